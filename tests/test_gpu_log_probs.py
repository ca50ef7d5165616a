"""Log probabilities, entropy, alternatives and their gradient against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2310_19509_amd as S
from oracle import lowp as L

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
INF = float("inf")


def _logits(seed, rows, cols, dtype, pad=0, masked=0.0, spread=3.0):
    rng = np.random.default_rng(seed)
    v = rng.standard_normal((rows, cols)) * spread
    v[rng.random((rows, cols)) < masked] = -np.inf
    buf = torch.full((rows, cols + pad), float("nan"), dtype=dtype, device="cuda")
    x = buf[:, :cols]
    x.copy_(torch.from_numpy(v))
    return x


def _targets(seed, rows, cols, n):
    t = np.random.default_rng(seed).integers(0, cols, (rows, n))
    if n > 1 and rows > 1:
        t[1, 0], t[1, 1] = -1, cols - 1
        t[0, 1] = t[0, 0]
    return torch.from_numpy(t).cuda()


def _score(x, t, k, stream=None):
    r, c = x.shape
    n = 0 if t is None else t.shape[1]
    new = lambda *s, dtype=torch.float32: torch.full(s, 77, dtype=dtype, device="cuda")  # noqa: E731
    logp, lse, ent, ids, top = new(r, n), new(r), new(r), new(r, k, dtype=torch.int64), new(r, k)
    b = S.sbn_log_probs_workspace(r, c, k)
    ws = torch.full((b,), 0xFF, dtype=torch.uint8, device="cuda") if b else None
    S.sbn_log_probs(x, t, k, logp, lse, ent, ids, top, workspace=ws, stream=stream)
    return [v.cpu().numpy() for v in (lse, logp, ent, ids, top)]


def _close(got, want, tol):
    both = np.isfinite(want)
    assert np.array_equal(got[~both], want[~both].astype(got.dtype), equal_nan=True)
    off = np.abs(got[both] - want[both])
    assert np.all(off <= np.broadcast_to(tol, want.shape)[both]), float((off / np.broadcast_to(tol, want.shape)[both]).max())


def _compare(x, t, k, got=None):
    got = got or _score(x, t, k)
    x64 = x.double().cpu().numpy()
    want = L.log_probs(x64, np.zeros((x.shape[0], 0), dtype=np.int64) if t is None else t.cpu().numpy(), k)
    # e^d in 32 bits: its argument is rounded twice (2^-23 of |d|, which its weight e^d keeps below 1 in every sum), its value a few times: 2^-21 of a sum
    # in all; log and the additions round at the size of the logits and of the
    # result, which is larger by log cols at most
    big = np.abs(np.where(np.isfinite(x64), x64, 0)).max()
    sum_rel = 2.0 ** -21
    _close(got[0], want[0], sum_rel + 2.0 ** -22 * (1 + big + np.log(x.shape[1])))
    _close(got[1], want[1], sum_rel + 2.0 ** -21 * (1 + big + np.abs(np.where(np.isfinite(want[1]), want[1], 0))))
    _close(got[2], want[2], 4 * sum_rel * (1 + np.abs(np.where(np.isfinite(want[2]), want[2], 0))) + 2.0 ** -22 * (1 + big + np.log(x.shape[1])))
    assert np.array_equal(got[3], want[3])
    _close(got[4], want[4], sum_rel + 2.0 ** -21 * (1 + big + np.abs(np.where(np.isfinite(want[4]), want[4], 0))))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,pad,n,k", [(1, 1, 0, 1, 1), (2, 3, 1, 2, 3), (3, 7, 0, 1, 0), (5, 8, 0, 1, 8), (4, 63, 2, 3, 20), (3, 64, 0, 1, 64), (2, 65, 1, 2, 64), (9, 511, 0, 1, 5),
                                               (3, 513, 3, 1, 64), (6, 2049, 0, 7, 20), (4, 8191, 1, 1, 50), (2, 8192, 0, 1, 1), (3, 8193, 0, 1, 64), (1, 50001, 7, 2, 20),
                                               (1100, 600, 0, 1, 5), (1030, 4100, 1, 1, 1), (1, 300000, 0, 1, 64)])
def test_against_64_bits(dtype, rows, cols, pad, n, k):
    _compare(_logits(rows + cols, rows, cols, dtype, pad), _targets(cols, rows, cols, n), k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,pad,n,k,masked", [(2049, 5, 0, 1, 5, 0.3), (2050, 700, 1, 2, 20, 0.0), (2051, 2050, 0, 1, 64, 0.5), (2048, 5001, 3, 70, 1, 0.98), (2048, 513, 0, 1, 0, 0.0)])
def test_many_rows(dtype, rows, cols, pad, n, k, masked):
    x = _logits(rows + cols, rows, cols, dtype, pad, masked)
    x[7] = -INF
    x[9, cols // 2] = float("nan")
    x[11] = torch.arange(cols, device="cuda") * 0.01
    x[13] = 2.0
    _compare(x, _targets(cols, rows, cols, n), k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols,pad,k,masked", [(16384, 0, 0, 0.0), (20003, 1, 0, 0.4), (28671, 0, 0, 0.0), (16391, 2, 5, 0.1), (33001, 1, 20, 0.2), (1201, 0, 64, 0.1), (1200, 0, 49, 0.98)])
def test_many_long_rows(dtype, cols, pad, k, masked):
    """Twelve rows over and over: the same bits wherever they lie, and those of 64 bits."""
    base, few = _logits(cols, 12, cols, dtype, 0, masked), _targets(cols, 12, cols, 2)
    base[7] = -INF
    base[9, cols // 2] = float("nan")
    base[10, cols - 1] = INF
    base[11] = torch.arange(cols, device="cuda") * 0.001
    pick = torch.arange(2050, device="cuda") % 12
    x = torch.empty(2050, cols + pad, dtype=dtype, device="cuda")[:, :cols]
    x.copy_(base[pick])
    got = _score(x, few[pick], k)
    for v in got:
        assert np.array_equal(v, v[:12][pick.cpu().numpy()], equal_nan=v.dtype != np.int64)
    _compare(base, few, k, [v[:12] for v in got])


@pytest.mark.parametrize("cols", [100, 5000, 40000])
@pytest.mark.parametrize("k", [1, 17, 64])
@pytest.mark.parametrize("kind", ["ascending", "descending", "equal", "zeros", "two values", "one", "few", "none", "low", "steps"])
def test_orders_ties_and_masks(cols, k, kind):
    """Rows that put aside as much as there is, rows of equal values, rows of which a mask leaves little or nothing."""
    i = torch.arange(cols, device="cuda", dtype=torch.float32)
    x = torch.empty(3, cols, device="cuda")
    if kind == "ascending":
        x[:] = i * 0.001
    elif kind == "descending":
        x[:] = -i * 0.001
    elif kind == "equal":
        x[:] = 1.25
    elif kind == "zeros":
        x[:] = torch.where(i % 3 == 0, -0.0, 0.0)
    elif kind == "two values":
        x[:] = (i % 97 == 5).float()
    elif kind == "one":
        x[:] = -INF
        x[:, cols // 2] = -4.0
    elif kind == "few":
        x[:] = -INF
        x[:, 3::cols // 9] = i[3::cols // 9] % 5
    elif kind == "none":
        x[:] = -INF
    elif kind == "low":
        x[:] = torch.finfo(torch.float32).min
        x[1, 7] = 0.0
    else:
        x[:] = torch.floor(i / 100)
    _compare(x, _targets(1, 3, cols, 2), k)


@pytest.mark.parametrize("cols", [40, 9000, 50000])
def test_nan_and_infinity_in_a_row(cols):
    x = _logits(3, 8, cols, torch.float32)
    x[1, 5] = float("nan")
    x[2, cols - 1] = INF
    x[3, 1], x[3, 7], x[3, 8] = INF, float("nan"), -float("nan")
    x[4, :] = float("nan")
    x[5, 9] = -INF
    x[6, 0], x[6, cols - 2] = INF, INF
    t = _targets(2, 8, cols, 2)
    t[2, 0] = cols - 1
    t[5, 0] = 9
    t[7, 0] = cols
    _compare(x, t, 10)


def test_masked_columns_with_the_types_lowest_value():
    for dtype in TYPES:
        x = _logits(5, 4, 3001, dtype)
        x[:, ::3] = torch.finfo(dtype).min
        x[2] = torch.finfo(dtype).min
        _compare(x, _targets(3, 4, 3001, 2), 20)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,pad,n,masked", [(1, 1, 0, 1, 0), (3, 9, 1, 2, 0.2), (2, 64, 0, 1, 0), (5, 2049, 2, 7, 0.3), (3, 10000, 0, 70, 0), (1, 40003, 0, 2, 0.9), (2100, 300, 0, 1, 0)])
@pytest.mark.parametrize("entropy", [False, True])
def test_gradient_formula(dtype, rows, cols, pad, n, masked, entropy):
    x, t = _logits(rows + cols, rows, cols, dtype, pad, masked), _targets(cols, rows, cols, n)
    if rows > 2:
        x[2] = -INF
    rng = np.random.default_rng(4)
    g, gh = rng.standard_normal((rows, n)).astype(np.float32), rng.standard_normal(rows).astype(np.float32) if entropy else None
    new = lambda *s: torch.empty(s, device="cuda")  # noqa: E731
    logp, lse, ent = new(rows, n), new(rows), new(rows)
    b = S.sbn_log_probs_workspace(rows, cols, 0)
    S.sbn_log_probs(x, t, 0, logp, lse, ent, workspace=torch.empty(b, dtype=torch.uint8, device="cuda") if b else None)
    grad = torch.full((rows, cols + pad), 7.0, dtype=dtype, device="cuda")
    gd, ghd = torch.from_numpy(g).cuda(), None if gh is None else torch.from_numpy(gh).cuda()
    S.sbn_log_probs_backward(x, t, lse, ent, gd, ghd, grad[:, :cols])
    assert (grad[:, cols:] == 7).all()
    x64 = x.double().cpu().numpy()
    want = L.log_probs_gradient(x64, t.cpu().numpy(), g.astype(np.float64), None if gh is None else gh.astype(np.float64))
    got = grad[:, :cols].double().cpu().numpy()
    half = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[dtype]
    # p and log p are off by 2^-20 (1 + |logits|) at most, which the factors of p and the target's own gradient scale
    lp = x64 - L.log_probs(x64, t.cpu().numpy(), 0)[0][:, None]
    p = np.where(np.isfinite(lp), np.exp(np.minimum(lp, 0)), 0)
    size = p * (np.abs(g).sum(1, keepdims=True) + (0 if gh is None else np.abs(gh)[:, None] * (np.abs(np.where(p > 0, lp, 0)) + np.log(cols) + 1)))
    tol = 2.0 ** -20 * 16 * size + np.abs(want) * half * 1.01 + 2.0 ** -22 * np.abs(g).sum(1, keepdims=True) * (want != 0) + (2.0 ** -24 if dtype == torch.float16 else 0)
    assert np.all(np.abs(got - want) <= tol), float((np.abs(got - want) - tol).max())
    again = x.clone() if pad == 0 else x
    S.sbn_log_probs_backward(again, t, lse, ent, gd, ghd, again)         # in the logits' place
    assert torch.equal(again, grad[:, :cols])


def test_gradient_against_differences():
    """Of the loss sum g logp + sum gh H, by central differences of the forward definition in 64 bits."""
    rows, cols, n = 3, 40, 2
    x, t = _logits(1, rows, cols, torch.float32, spread=1.5), _targets(6, rows, cols, n)
    rng = np.random.default_rng(2)
    g, gh = rng.standard_normal((rows, n)), rng.standard_normal(rows)
    loss = lambda v: (lambda o: (g * o[1]).sum() + (gh * o[2]).sum())(L.log_probs(v, t.cpu().numpy(), 0))  # noqa: E731
    x64, h = x.double().cpu().numpy(), 1e-5
    want = np.zeros_like(x64)
    for i in np.ndindex(*x64.shape):
        a, b = x64.copy(), x64.copy()
        a[i] += h
        b[i] -= h
        want[i] = (loss(a) - loss(b)) / (2 * h)
    logp, lse, ent = torch.empty(rows, n, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    S.sbn_log_probs(x, t, 0, logp, lse, ent)
    grad = torch.empty_like(x)
    f = lambda v: torch.from_numpy(v.astype(np.float32)).cuda()  # noqa: E731
    S.sbn_log_probs_backward(x, t, lse, ent, f(g), f(gh), grad)
    # the differences' own error: h^2 / 6 of third derivatives of order 1, and 1e-16 * 10 / h
    assert np.abs(grad.double().cpu().numpy() - want).max() <= 1e-5


def test_rows_far_apart():
    ld = 3 << 29
    x = torch.empty(2 * ld + 70000, dtype=torch.bfloat16, device="cuda").as_strided((3, 5001), (ld, 1))
    x.copy_(_logits(1, 3, 5001, torch.bfloat16))
    t = _targets(1, 3, 5001, 2)
    _compare(x, t, 9)
    lse = torch.from_numpy(_score(x, t, 0)[0]).cuda()
    g = torch.ones(3, 2, device="cuda")
    want = torch.empty(3, 5001, dtype=torch.bfloat16, device="cuda")
    S.sbn_log_probs_backward(x.clone(memory_format=torch.contiguous_format), t, lse, None, g, None, want)
    S.sbn_log_probs_backward(x, t, lse, None, g, None, x)
    assert torch.equal(x, want)


def test_streams_no_rows_and_refusals():
    x, t = _logits(2, 3, 20000, torch.bfloat16), _targets(2, 3, 20000, 1)
    want = _score(x, t, 5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _score(x, t, 5)
    assert all(np.array_equal(a, b) for a, b in zip(got, want))
    e = torch.empty
    S.sbn_log_probs(x[:0], t[:0], 5, e(0, 1, device="cuda"), e(0, device="cuda"), None, e(0, 5, device="cuda", dtype=torch.int64), e(0, 5, device="cuda"))
    lse, logp, ids, top = e(3, device="cuda"), e(3, 1, device="cuda"), e(3, 5, device="cuda", dtype=torch.int64), e(3, 5, device="cuda")
    ws = e(S.sbn_log_probs_workspace(3, 20000, 5), dtype=torch.uint8, device="cuda")
    for bad in (lambda: S.sbn_log_probs(x, t.int(), 5, logp, lse, None, ids, top, ws), lambda: S.sbn_log_probs(x, t[:2], 5, logp, lse, None, ids, top, ws),
                lambda: S.sbn_log_probs(x, t, 5, logp, lse, None, ids.int(), top, ws), lambda: S.sbn_log_probs(x, t, 4, logp, lse, None, ids, top, ws),
                lambda: S.sbn_log_probs(x.double(), t, 5, logp, lse, None, ids, top, ws), lambda: S.sbn_log_probs(x, t, 5, logp, None, None, ids, top, ws),
                lambda: S.sbn_log_probs_backward(x, t, lse, None, logp, lse, x), lambda: S.sbn_log_probs_backward(x, t, lse, lse, logp, lse, x.float())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: S.sbn_log_probs(x, t, 5, logp, lse, None, ids, top), lambda: S.sbn_log_probs(x, t, 5, logp, lse, None, ids, top, ws[:-16])):
        with pytest.raises(S.SbnError):
            bad()
