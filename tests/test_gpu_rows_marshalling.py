"""The calls over rows give the same through the marshalling module and through the Python code, which serves what the module leaves to it."""
import numpy as np
import pytest
import torch

import paper_2310_19509_amd as S
from paper_2310_19509_amd import _lib, api

pytestmark = pytest.mark.gpu


def _everything():
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(37, 333, device="cuda", generator=g, dtype=torch.float32).bfloat16()[:, :300]
    r = torch.randn(37, 300, device="cuda", generator=g)
    w = torch.randn(300, device="cuda", generator=g)
    out = []
    for fmt in (S.SBN_MXFP4, S.SBN_MXFP8, S.SBN_FP8_ROW):
        c, s = S.sbn_quantized_empty(fmt, 37, 300)
        S.sbn_quantize(x, fmt, c, s)
        y = torch.empty(37, 300, device="cuda")
        S.sbn_dequantize(c, s, fmt, y)
        out += [c.clone(), s.clone(), y]
        total, n = torch.empty_like(r), torch.empty(37, 300, device="cuda", dtype=torch.bfloat16)
        S.sbn_add_rmsnorm(x, w, 1e-6, residual=r, total=total, y=n, fmt=fmt, codes=c, scales=s)
        out += [c.clone(), s.clone(), total, n]
        S.sbn_add_rmsnorm(x, None, 1e-6, fmt=fmt, codes=c, scales=s)
        p = S.sbn_mx_pack(np.random.default_rng(1).standard_normal((50, 300)).astype(np.float32))
        z = torch.empty(37, 50, device="cuda", dtype=torch.float16)
        b = S.sbn_linear_mx_workspace(p, fmt, 37)
        S.sbn_linear_mx(p, c, s, fmt, z, workspace=torch.empty(b, device="cuda", dtype=torch.uint8) if b else None)
        out += [c, s, z]
    t = torch.randint(-1, 300, (37, 3), device="cuda", generator=g)
    for k in (0, 7):
        e = lambda *v, dtype=torch.float32: torch.empty(v, device="cuda", dtype=dtype)  # noqa: E731
        logp, lse, ent, ids, top = e(37, 3), e(37), e(37), e(37, k, dtype=torch.int64) if k else None, e(37, k) if k else None
        S.sbn_log_probs(x, t, k, logp, lse, ent, ids, top)
        grad = torch.empty(37, 300, device="cuda", dtype=torch.bfloat16)
        S.sbn_log_probs_backward(x, t, lse, ent, logp, lse, grad)
        out += [logp, lse, ent, grad] + ([ids, top] if k else [])
        S.sbn_log_probs_backward(x, t, lse, None, logp, None, grad := torch.empty_like(grad))
        out.append(grad)
    S.sbn_log_probs(x, None, 0, None, lse)
    return out + [lse]


def test_both_ways_give_the_same(monkeypatch):
    assert _lib.marshal() is not None
    a = _everything()
    monkeypatch.setattr(api, "_rows_native", (None,))
    b = _everything()
    assert len(a) == len(b) and all(torch.equal(u.nan_to_num(7.0) if u.is_floating_point() else u, v.nan_to_num(7.0) if v.is_floating_point() else v) for u, v in zip(a, b))


def test_the_module_takes_ordinary_calls():
    m = _lib.marshal()
    x = torch.randn(4, 64, device="cuda")
    c, s = S.sbn_quantized_empty(S.SBN_MXFP4, 4, 64)
    assert m.quantize(x, S.SBN_MXFP4, c, s, None) == 0
    assert m.dequantize(c, s, S.SBN_MXFP4, x, None) == 0
    assert m.norm(x, None, 1e-6, None, None, None, S.SBN_MXFP4, c, s, None) == 0
    p = S.sbn_mx_pack(np.ones((8, 64), dtype=np.float32))
    assert m.linear(p, c, s, S.SBN_MXFP4, torch.empty(4, 8, device="cuda"), None, None) == 0
    lse, t, one = torch.empty(4, device="cuda"), torch.zeros(4, 1, dtype=torch.int64, device="cuda"), torch.empty(4, 1, device="cuda")
    assert m.score(x, t, 0, one, lse, None, None, None, None, None) == 0
    assert m.backward(x, t, lse, None, one, None, x, None) == 0
    # what it leaves to the Python code: other streams, types, shapes, strides
    assert m.quantize(x, S.SBN_MXFP4, c, s, torch.cuda.Stream()) is None
    assert m.quantize(x.double(), S.SBN_MXFP4, c, s, None) is None
    assert m.quantize(x.t(), S.SBN_MXFP4, c, s, None) is None
    assert m.quantize(x, S.SBN_MXFP8, c, s, None) is None
    assert m.quantize(x.cpu(), S.SBN_MXFP4, c, s, None) is None
    assert m.linear(p, c, s, S.SBN_MXFP4, torch.empty(4, 7, device="cuda"), None, None) is None
    assert m.score(x, t.int(), 0, one, lse, None, None, None, None, None) is None
    assert m.backward(x, t, lse, None, one, lse, x, None) is None
