"""4-bit weights on the host: the packer against the definition, and what the calls refuse without a GPU."""
import numpy as np
import pytest

import paper_2310_19509_amd as S
from oracle import lowp as L


def _bytes(seed, *shape):
    return np.random.default_rng(seed).integers(0, 256, shape, dtype=np.uint8)


def _w(seed, n, k, spread=6.0):
    rng = np.random.default_rng(seed)
    w = rng.standard_normal((n, k)) * np.exp2(rng.uniform(-spread, spread, (n, 1)))
    w[rng.random((n, k)) < 0.05] = 0.0
    return w.astype(np.float32)


@pytest.mark.parametrize("n,k", [(1, 1), (3, 31), (16, 32), (17, 33), (40, 200), (5, 513)])
def test_pack_quantises_by_the_definition(n, k):
    w = _w(n * 1000 + k, n, k)
    codes, scales, bias = S.sbn_mx_unpack(S.sbn_mx_pack(w, device=-1))
    want_c, want_s = L.quantize(w.astype(np.float64), L.MXFP4)
    assert np.array_equal(codes, want_c) and np.array_equal(scales, want_s) and not bias.any()


def test_ties_saturation_tiny_and_huge_blocks():
    v = np.array([0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 7.99, 0.2499, 0.2501, 4.999, 5.001, -0.25, -0.75, -5.0, -7.5, -0.0, 6.0], dtype=np.float32)
    rows = [v * np.float32(s) for s in (1.0, 2.0 ** -100, 2.0 ** 100, 2.0 ** -126, 2.0 ** 125 / 8)] + [np.zeros_like(v), v * 0 + np.float32(1e-45)]
    w = np.stack(rows)
    codes, scales, _ = S.sbn_mx_unpack(S.sbn_mx_pack(w, device=-1))
    want_c, want_s = L.quantize(w.astype(np.float64), L.MXFP4)
    assert np.array_equal(codes, want_c) and np.array_equal(scales, want_s)


def test_pack_applies_mask_and_orders():
    rng = np.random.default_rng(3)
    n, k, go, gi = 24, 40, 8, 2
    w, bias = _w(4, n, k), rng.standard_normal(n).astype(np.float32)
    po, pi = rng.permutation(n).astype(np.int32), rng.permutation(k).astype(np.int32)
    mask = (rng.random((n // go, k // gi)) < 0.5).astype(np.uint8)
    p = S.sbn_mx_pack(w, go, gi, mask=mask, bias=bias, perm_out=po, perm_in=pi, act=S.SBN_ACT_RELU, device=-1)
    want = w[po][:, pi] * np.kron(mask, np.ones((go, gi)))
    want_c, want_s = L.quantize(want, L.MXFP4)
    codes, scales, b = S.sbn_mx_unpack(p)
    # (a removed weight is +0 whatever its sign was)
    assert np.array_equal(L.values(codes, scales, L.MXFP4, k), L.values(want_c, want_s, L.MXFP4, k))
    assert np.array_equal(scales, want_s) and np.array_equal(b, bias[po])
    assert S.sbn_mx_info(p) == dict(c_in=k, c_out=n, act=S.SBN_ACT_RELU, device=-1, device_bytes=0)


@pytest.mark.parametrize("k", [32, 33, 63])
def test_codes_go_in_and_come_out(k):
    n, blocks = 19, (k + 31) // 32
    codes, scales = _bytes(1, n, blocks * 16), _bytes(2, n, blocks)
    bias = np.arange(n, dtype=np.float32)
    c, s, b = S.sbn_mx_unpack(S.sbn_mx_pack_codes(codes, scales, k, bias=bias, device=-1))
    want = codes.copy()
    for i in range(k, blocks * 32):
        want[:, i // 2] &= 0x0F if i & 1 else 0xF0
    assert np.array_equal(c, want) and np.array_equal(s, np.where(scales > 252, 255, scales)) and np.array_equal(b, bias)


def _error(fn):
    with pytest.raises(S.SbnError) as e:
        fn()
    return e.value.code


def test_pack_refuses():
    w = _w(1, 8, 8)
    bad = w.copy()
    bad[3, 3] = np.nan
    assert _error(lambda: S.sbn_mx_pack(bad, device=-1)) == -1
    bad[3, 3] = np.inf
    assert _error(lambda: S.sbn_mx_pack(bad, device=-1)) == -1
    assert _error(lambda: S.sbn_mx_pack(w, act=7, device=-1)) == -1
    assert _error(lambda: S.sbn_mx_pack(w, device=-2)) == -1
    assert _error(lambda: S.sbn_mx_pack(w, 5, 4, mask=np.ones((1, 2)), device=-1)) == -1
    assert _error(lambda: S.sbn_mx_pack(_w(1, 10, 8), 4, 4, mask=np.ones((3, 2)), device=-1)) == -2
    assert _error(lambda: S.sbn_mx_pack(w, perm_out=np.zeros(8), device=-1)) == -3
    with pytest.raises(ValueError):
        S.sbn_mx_pack_codes(_bytes(1, 4, 16), _bytes(1, 4, 2), 32, device=-1)
    with pytest.raises(ValueError):
        S.sbn_mx_pack_codes(_bytes(1, 4, 16), _bytes(1, 4, 1), 32, bias=np.zeros(3, dtype=np.float32), device=-1)


def test_run_calls_refuse_before_any_launch():
    from paper_2310_19509_amd import _lib
    l = _lib.lib()
    p = S.sbn_mx_pack(_w(1, 8, 8), device=-1)
    a = 1 << 20                                          # an aligned address that no call here gets to use
    assert l.sbn_linear_mx(p.handle, a, a, S.SBN_MXFP4, 1, a, S.SBN_F32, 8, None, 0, None) == -6
    assert l.sbn_linear_mx(None, a, a, S.SBN_MXFP4, 1, a, S.SBN_F32, 8, None, 0, None) == -1
    assert l.sbn_linear_mx(p.handle, a, a, 9, 1, a, S.SBN_F32, 8, None, 0, None) == -1
    for bad in (dict(fmt=3), dict(t=7), dict(rows=-1), dict(cols=0), dict(cols=1 << 31), dict(ld=7), dict(x=None), dict(x=a + 1), dict(codes=a + 8), dict(scales=None)):
        v = dict(x=a, t=S.SBN_BF16, rows=2, cols=8, ld=8, fmt=S.SBN_MXFP4, codes=a, scales=a) | bad
        assert l.sbn_quantize(v["x"], v["t"], v["rows"], v["cols"], v["ld"], v["fmt"], v["codes"], v["scales"], None) == -1, bad
        assert l.sbn_dequantize(v["codes"], v["scales"], v["fmt"], v["rows"], v["cols"], v["x"], v["t"], v["ld"], None) == -1, bad
    assert l.sbn_quantize(a, S.SBN_BF16, 2, 8, 8, S.SBN_FP8_ROW, a, a + 2, None) == -1
    assert l.sbn_quantize(None, S.SBN_F32, 0, 8, 8, S.SBN_MXFP4, None, None, None) == 0
    assert "columns" in S.sbn_last_error() or S.sbn_last_error() == ""

    def score(**bad):
        v = dict(x=a, t=S.SBN_F32, rows=2, cols=100, ld=100, targets=a, n=1, k=5, logp=a, lse=a, entropy=None, ids=a, top=a, ws=None, wb=0) | bad
        return l.sbn_log_probs(v["x"], v["t"], v["rows"], v["cols"], v["ld"], v["targets"], v["n"], v["k"], v["logp"], v["lse"], v["entropy"], v["ids"], v["top"],
                               v["ws"], v["wb"], None)
    for bad in (dict(x=None), dict(t=5), dict(rows=-2), dict(cols=0), dict(ld=99), dict(targets=None), dict(n=-1), dict(k=-1), dict(k=65), dict(cols=4, ld=4),
                dict(logp=None), dict(lse=None), dict(ids=None), dict(top=None), dict(ids=a + 4), dict(lse=a + 1), dict(cols=1 << 20, ld=1 << 20, rows=1)):
        assert score(**bad) == -1, bad
    assert score(rows=0) == 0

    def back(**bad):
        v = dict(x=a, t=S.SBN_F32, rows=2, cols=100, ld=100, targets=a, n=1, lse=a, entropy=a, g=a, gh=a, grad=a, ldg=100) | bad
        return l.sbn_log_probs_backward(v["x"], v["t"], v["rows"], v["cols"], v["ld"], v["targets"], v["n"], v["lse"], v["entropy"], v["g"], v["gh"], v["grad"], v["ldg"], None)
    for bad in (dict(x=None), dict(t=5), dict(rows=-2), dict(cols=0), dict(ld=99), dict(ldg=99), dict(ldg=101), dict(targets=None), dict(g=None), dict(lse=None),
                dict(entropy=None), dict(grad=None)):
        assert back(**bad) == -1, bad

    def norm(**bad):
        v = dict(rows=2, cols=8, x=a, x_type=S.SBN_BF16, ldx=8, residual=a, r_type=S.SBN_BF16, ldr=8, total=a, ldt=8, weight=a, eps=1e-6, y=a + 4096, ldy=8, format=0) | bad
        r = _lib.RmsNorm()
        for f, x in v.items():
            setattr(r, f, x)
        return l.sbn_add_rmsnorm(r, None)
    for bad in (dict(rows=-1), dict(cols=0), dict(x=None), dict(x_type=4), dict(ldx=7), dict(r_type=S.SBN_F16), dict(ldr=7), dict(ldt=9), dict(total=a + 1), dict(residual=None),
                dict(weight=a + 2), dict(eps=-1.0), dict(eps=float("nan")), dict(y=a), dict(y=None, total=None), dict(format=2), dict(format=S.SBN_MXFP4),
                dict(format=S.SBN_MXFP4, codes=a + 4, scales=a)):
        assert norm(**bad) == -1, bad
    assert l.sbn_add_rmsnorm(None, None) == -1
    assert norm(rows=0) == 0


def test_sizes():
    assert S.sbn_quantized_bytes(S.SBN_MXFP4, 3, 33) == (3 * 32, 6)
    assert S.sbn_quantized_bytes(S.SBN_MXFP8, 3, 33) == (3 * 64, 6)
    assert S.sbn_quantized_bytes(S.SBN_FP8_ROW, 3, 33) == (3 * 64, 12)
    assert _error(lambda: S.sbn_quantized_bytes(1, 3, 33)) == -1
    assert S.sbn_log_probs_workspace(4096, 50000, 5) == 0 and S.sbn_log_probs_workspace(1, 100000, 5) > 0


def test_sizes_that_pass_64_bits_are_refused():
    for rows, cols in [(1 << 40, 1 << 21), (1 << 31, 1 << 30), ((1 << 40) + 1, 1)]:
        assert _error(lambda: S.sbn_quantized_bytes(S.SBN_MXFP8, rows, cols)) == -1
        assert _error(lambda: S.sbn_log_probs_workspace(rows, cols, 5)) == -1
    assert S.sbn_quantized_bytes(S.SBN_MXFP8, 1 << 30, 1 << 20)[0] == 1 << 50
