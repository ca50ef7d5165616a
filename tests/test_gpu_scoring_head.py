"""The example's layers together, against the definitions in 64 bits; eager and as a HIP graph."""
import os
import sys

import numpy as np
import pytest
import torch

import paper_2310_19509_amd as S
from oracle import lowp as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))
pytestmark = pytest.mark.gpu


def _np(t):
    return t.double().cpu().numpy()


def _product(y, codes, scales, fmt, w, relu):
    """bfloat16 results: their rounding, the multiplies' cut of 2^-13 of the products' size and as much for sums in 32 bits."""
    n = L.values(codes.cpu().numpy(), scales.cpu().numpy(), fmt, w.shape[1])
    want = n @ w.T
    tol = np.abs(want) * 2.0 ** -8 * 1.01 + 2.0 ** -12 * (np.abs(n) @ np.abs(w).T)
    assert np.all(np.abs(_np(y) - (np.maximum(want, 0) if relu else want)) <= tol)


@pytest.mark.parametrize("rows,hidden,vocab,fmt,sparsity", [(1, 256, 1000, S.SBN_MXFP8, 0), (37, 128, 333, S.SBN_FP8_ROW, 50), (300, 256, 2001, S.SBN_MXFP4, 0)])
def test_example_layer_by_layer(rows, hidden, vocab, fmt, sparsity):
    """The example's calls one by one, each output against the definition applied to the call's own inputs; then the example itself: the same bits."""
    from scoring_head import ScoringHead
    from test_gpu_lowp_rows import NORM_REL, _check_codes
    head = ScoringHead(rows, hidden, 2, vocab, top=5, fmt=fmt, sparsity=sparsity)
    g = torch.Generator(device="cuda").manual_seed(5)
    x0, start = (torch.randn(rows, hidden, device="cuda", generator=g).bfloat16() for _ in range(2))
    targets = torch.randint(0, vocab, (rows, 1), device="cuda", generator=g)
    wv = []
    for w, mask in head.weights:
        w = w.reshape(w.shape[0], -1).astype(np.float64)
        if mask is not None:
            w = w * np.kron(mask, np.ones((4, 4)))
        wv.append(L.values(*L.quantize(w, L.MXFP4), L.MXFP4, w.shape[1]))

    x, residual = x0, start.clone()

    def norm(weight):
        total = x.float() + residual.float()
        S.sbn_add_rmsnorm(x, weight, 1e-6, residual=residual, total=residual, fmt=fmt, codes=head.narrow[0], scales=head.narrow[1])
        assert torch.equal(residual, total.bfloat16())
        _check_codes(*head.narrow, fmt, L.rmsnorm(_np(total), _np(weight), 1e-6), NORM_REL)

    for b, (up, down) in enumerate(head.blocks):
        norm(head.norms[b])
        S.sbn_linear_mx(up, *head.narrow, fmt, head.up, workspace=head.workspace)
        _product(head.up, *head.narrow, fmt, wv[2 * b], True)
        S.sbn_quantize(head.up, fmt, *head.wide)
        codes, scales = L.quantize(_np(head.up), fmt)
        assert np.array_equal(head.wide[0].cpu().numpy(), codes) and np.array_equal(head.wide[1].cpu().numpy(), scales)
        S.sbn_linear_mx(down, *head.wide, fmt, head.down, workspace=head.workspace)
        _product(head.down, *head.wide, fmt, wv[2 * b + 1], False)
        x = head.down
    norm(head.norms[-1])
    S.sbn_linear_mx(head.head, *head.narrow, fmt, head.logits, workspace=head.workspace)
    _product(head.logits, *head.narrow, fmt, wv[-1], False)
    logits, last = head.logits.clone(), residual

    residual = start.clone()
    logp, entropy, ids, top = head.run(x0, residual, targets)
    assert torch.equal(head.logits, logits) and torch.equal(residual, last)
    lse, lp, ent, order, tl = L.log_probs(_np(logits), targets.cpu().numpy(), 5)
    assert np.array_equal(ids.cpu().numpy(), order)
    assert np.allclose(_np(logp), lp, atol=1e-5) and np.allclose(_np(entropy), ent, atol=1e-5) and np.allclose(_np(top), tl, atol=1e-5)


def test_a_graph_of_the_example_gives_the_same_on_every_replay():
    from scoring_head import ScoringHead
    rows, hidden, vocab = 20, 512, 30000
    head = ScoringHead(rows, hidden, 2, vocab)
    x, start = (torch.randn(rows, hidden, device="cuda").bfloat16() for _ in range(2))
    targets = torch.randint(0, vocab, (rows, 1), device="cuda")
    residual = start.clone()
    want = [t.clone() for t in (*head.run(x, residual, targets), residual)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        residual.copy_(start)
        head.run(x, residual, targets)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        residual.copy_(start)
        got = head.run(x, residual, targets)
    for _ in range(4):
        for t in (*got, residual):
            t.zero_()
        torch.randn(1000, 1000, device="cuda").sum()                     # the program's own work in between
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*got, residual), want))


def test_a_classifiers_logits():
    """A chain's float32 logits, as they come out of a network."""
    rng = np.random.default_rng(1)
    p = S.sbn_pack(S.SBN_CONV1X1, (rng.standard_normal((1000, 1, 1, 1024)) * 0.05).astype(np.float32), 4, 4)
    c = S.sbn_chain_create([S.sparse_item(p)])
    x = torch.rand(16, 1, 1, 1024, device="cuda")
    y = torch.empty(16, 1, 1, 1000, device="cuda")
    S.sbn_pointwise_chain(c, x, y, 16, 1, 1, None)
    logits = y.view(16, 1000)
    new = lambda *s, dtype=torch.float32: torch.empty(s, dtype=dtype, device="cuda")  # noqa: E731
    lse, ids, top = new(16), new(16, 5, dtype=torch.int64), new(16, 5)
    S.sbn_log_probs(logits, None, 5, None, lse, None, ids, top)
    want = L.log_probs(_np(logits), np.zeros((16, 0), dtype=np.int64), 5)
    assert np.array_equal(ids.cpu().numpy(), want[3]) and np.allclose(_np(top), want[4], atol=1e-5) and np.allclose(_np(lse), want[0], atol=1e-5)
