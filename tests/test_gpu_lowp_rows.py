"""Rows into 4 and 8 bits and back, and the norm with the residual's addition, against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2310_19509_amd as S
from oracle import lowp as L

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
FORMATS = [S.SBN_MXFP4, S.SBN_MXFP8, S.SBN_FP8_ROW]
# half a unit in the last place over the least value of its binade: 2^-(significant bits)
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def _x(seed, rows, cols, dtype, pad=0, offset=0):
    """Rows of very different size with exact ties, zeros and outliers; a view into a wider buffer that begins `offset` elements in."""
    rng = np.random.default_rng(seed)
    v = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-6, 6, (rows, 1)))
    tie = rng.random((rows, cols)) < 0.3
    v = np.where(tie, np.round(v * 8) / 8, v)
    v[rng.random((rows, cols)) < 0.02] *= 30
    v[rng.random((rows, cols)) < 0.05] = 0.0
    if rows > 2:
        v[rows // 2] = 0.0
    buf = torch.full((rows * (cols + pad) + offset + 8,), float("nan"), dtype=dtype, device="cuda")
    x = buf[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    x.copy_(torch.from_numpy(v))
    return x


def _np(t):
    return t.double().cpu().numpy()


def _quantize(x, fmt):
    codes, scales = S.sbn_quantized_empty(fmt, *x.shape)
    codes.fill_(0xAA)
    S.sbn_quantize(x, fmt, codes, scales)
    return codes, scales


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows,cols,pad,offset", [(1, 1, 0, 0), (1, 7, 0, 1), (3, 8, 0, 0), (5, 31, 2, 3), (4, 32, 0, 0), (2, 33, 1, 0), (300, 70, 3, 1), (7, 2048, 0, 0),
                                                  (1025, 129, 0, 0), (1030, 2047, 1, 0), (3, 8195, 5, 1), (2, 40000, 0, 0)])
def test_quantize_is_bit_exact(dtype, fmt, rows, cols, pad, offset):
    x = _x(rows * 7 + cols, rows, cols, dtype, pad, offset)
    codes, scales = _quantize(x, fmt)
    want_c, want_s = L.quantize(_np(x), fmt)
    assert np.array_equal(scales.cpu().numpy(), want_s)
    assert np.array_equal(codes.cpu().numpy(), want_c)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (3, 31, 2), (5, 64, 0), (200, 77, 1), (3, 4099, 0)])
def test_dequantize_rounds_the_value_once(dtype, fmt, rows, cols, pad):
    x = _x(rows + cols, rows, cols, torch.float32)
    codes, scales = _quantize(x, fmt)
    y = torch.full((rows, cols + pad), 7.0, dtype=dtype, device="cuda")
    S.sbn_dequantize(codes, scales, fmt, y[:, :cols])
    want = L.values(codes.cpu().numpy(), scales.cpu().numpy(), fmt, cols)
    # blocks: element times a power of two is exact in 32 bits.  rows: the product rounds to 32 bits first
    got = _np(y[:, :cols])
    if fmt == S.SBN_FP8_ROW:
        assert np.all(np.abs(got - want) <= np.abs(want) * (HALF_ULP[dtype] + 2.0 ** -24) * 1.001 + 2.0 ** -24 * (dtype == torch.float16))
    else:
        assert np.array_equal(got, _np(torch.from_numpy(want).to(dtype)))
    assert (y[:, cols:] == 7).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_every_code_is_its_value(fmt):
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").repeat(1, 2).reshape(1, 512)
    cols = 1024 if fmt == S.SBN_MXFP4 else 512
    scales = torch.tensor([0.75], device="cuda") if fmt == S.SBN_FP8_ROW else torch.arange(100, 100 + cols // 32, dtype=torch.uint8, device="cuda")[None]
    y = torch.empty(1, cols, device="cuda")
    S.sbn_dequantize(codes, scales, fmt, y)
    want = L.values(codes.cpu().numpy(), scales.cpu().numpy(), fmt, cols)
    assert np.array_equal(_np(y), want, equal_nan=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fmt", FORMATS)
def test_extreme_rows(dtype, fmt):
    """Zeros, the type's smallest and largest values, NaN and infinities, each in a row of its own."""
    top, tiny = torch.finfo(dtype).max, torch.finfo(dtype).smallest_normal
    rows = [0.0, tiny, top, -top, float("nan"), float("inf"), -float("inf")]
    x = torch.randn(len(rows), 100, device="cuda").clamp(-3, 3).mul(0.01).to(dtype)
    for i, v in enumerate(rows):
        if v == 0 or v == tiny:
            x[i] = 0
        x[i, 40] = v
    codes, scales = _quantize(x, fmt)
    y = torch.empty(len(rows), 100, device="cuda")
    S.sbn_dequantize(codes, scales, fmt, y)
    got = _np(y)
    want_c, want_s = L.quantize(_np(x[:4]), fmt)
    assert np.array_equal(codes[:4].cpu().numpy(), want_c) and np.array_equal(scales[:4].cpu().numpy(), want_s)
    for i in (4, 5, 6):
        if fmt == S.SBN_FP8_ROW:
            assert np.isnan(got[i]).all() and torch.isnan(scales[i])
        else:
            assert np.isnan(got[i, 32:64]).all() and scales[i, 1] == 255 and np.isfinite(got[i, :32]).all() and np.isfinite(got[i, 64:]).all()


def _check_codes(codes, scales, fmt, y, rel):
    """Codes of values that are known to `rel`: each is within half a step (of the scale that was chosen) of the value, the scale of
    the block is the one of a largest magnitude within `rel`."""
    codes, scales = codes.cpu().numpy(), scales.cpu().numpy()
    rows, cols = y.shape
    got = L.values(codes, scales, fmt, cols)
    top_el = 6.0 if fmt == S.SBN_MXFP4 else 448.0
    if fmt == S.SBN_FP8_ROW:
        a = np.abs(y).max(1)
        assert np.all(np.abs(scales - a / 448) <= a / 448 * (rel + 2.0 ** -23))
        s = np.repeat(scales[:, None].astype(np.float64), cols, 1)
    else:
        n = -(-cols // 32)
        p = np.zeros((rows, n * 32))
        p[:, :cols] = np.abs(y)
        a = p.reshape(rows, n, 32).max(2)
        assert np.all((scales == L.block_bytes(a * (1 - rel), fmt)) | (scales == L.block_bytes(a * (1 + rel), fmt)))
        s = np.repeat(np.exp2(scales.astype(np.float64) - 127), 32, 1)[:, :cols]
    v = np.minimum(np.abs(y), top_el * s) / np.where(s > 0, s, 1)
    least, mantissa = (0, 1) if fmt == S.SBN_MXFP4 else (-6, 3)
    _, e = np.frexp(np.maximum(v, 2.0 ** least))
    step = np.exp2(e - 1.0 - mantissa)
    off = np.abs(np.abs(got) / np.where(s > 0, s, 1) - v)
    assert np.all(off <= step / 2 + 2 * (rel + 2.0 ** -23) * v + 1e-30)
    assert np.all((got * y >= 0))


# y = h w / rms: the sum of squares is 32 bits with at most 64 additions in a row (2^-19 of it, half that in the root), the rest adds single roundings
NORM_REL = 2.0 ** -20 + 2.0 ** -23


@pytest.mark.parametrize("xt,rt", [(torch.float32, None), (torch.float32, torch.float32), (torch.bfloat16, None), (torch.bfloat16, torch.bfloat16),
                                   (torch.bfloat16, torch.float32), (torch.float16, None), (torch.float16, torch.float16), (torch.float16, torch.float32)])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (3, 31, 1), (2, 64, 0), (1040, 100, 0), (1025, 2048, 0), (5, 4096, 0), (600, 4101, 3), (3, 8192, 0), (4, 20001, 0), (2, 33001, 7)])
def test_norm(xt, rt, rows, cols, pad):
    x = _x(rows + cols, rows, cols, xt, pad, 1)
    r = None if rt is None else _x(rows + cols + 1, rows, cols, rt, pad, 1)
    w = torch.randn(cols, device="cuda") if cols % 2 else None
    total = None if r is None else torch.empty(rows, cols + pad, dtype=rt, device="cuda")[:, :cols]
    h32 = x.float() if r is None else x.float() + r.float()
    want = L.rmsnorm(_np(h32), None if w is None else _np(w), 1e-5)
    for fmt in (0, *FORMATS):
        y = torch.empty(rows, cols + pad, dtype=xt, device="cuda")[:, :cols] if fmt in (0, S.SBN_MXFP8) else None
        codes, scales = S.sbn_quantized_empty(fmt, rows, cols) if fmt else (None, None)
        S.sbn_add_rmsnorm(x, w, 1e-5, residual=r, total=total, y=y, fmt=fmt, codes=codes, scales=scales)
        if r is not None:
            assert torch.equal(total, h32.to(rt))
        if y is not None:
            got = _np(y)
            assert np.all(np.abs(got - want) <= np.abs(want) * (NORM_REL + HALF_ULP[xt] * 1.01) + (2.0 ** -24 if xt == torch.float16 else 1e-37))
        if fmt:
            _check_codes(codes, scales, fmt, want, NORM_REL)


@pytest.mark.parametrize("cols", [500, 5000, 40000])
@pytest.mark.parametrize("where", ["residual", "x"])
def test_norm_in_place(cols, where):
    rows = 1100 if cols == 500 else 9
    x, r = _x(1, rows, cols, torch.bfloat16), _x(2, rows, cols, torch.bfloat16)
    want_total = torch.empty_like(x, memory_format=torch.contiguous_format)
    c0, s0 = S.sbn_quantized_empty(S.SBN_FP8_ROW, rows, cols)
    S.sbn_add_rmsnorm(x, None, 1e-6, residual=r, total=want_total, fmt=S.SBN_FP8_ROW, codes=c0, scales=s0)
    c1, s1 = S.sbn_quantized_empty(S.SBN_FP8_ROW, rows, cols)
    to = r if where == "residual" else x
    S.sbn_add_rmsnorm(x, None, 1e-6, residual=r, total=to, fmt=S.SBN_FP8_ROW, codes=c1, scales=s1)
    assert torch.equal(to, want_total) and torch.equal(c0, c1) and torch.equal(s0, s1)


def test_norm_of_zero_nan_infinite_and_huge_rows():
    x = torch.randn(5, 3000, device="cuda")
    x[0] = 0
    x[1, 7] = float("nan")
    x[2, 8] = float("inf")
    x[3] = 1e30
    y = torch.empty_like(x)
    codes, scales = S.sbn_quantized_empty(S.SBN_FP8_ROW, 5, 3000)
    S.sbn_add_rmsnorm(x, None, 0.0, y=y, fmt=S.SBN_FP8_ROW, codes=codes, scales=scales)
    # 0 / sqrt(0): the root is infinite and zeros give NaN unless eps is there
    assert torch.isnan(y[1]).all() and torch.isnan(y[2, 8]) and torch.isnan(scales[1:3]).all()
    assert (y[3] == 0).all() and scales[3] == 0 and torch.isfinite(y[4]).all()
    S.sbn_add_rmsnorm(x, None, 1e-6, y=y, fmt=S.SBN_FP8_ROW, codes=codes, scales=scales)
    assert (y[0] == 0).all() and scales[0] == 0 and (codes[0] == 0).all()


@pytest.mark.parametrize("rows,cols,xt,rt", [(2048, 4096, torch.bfloat16, torch.bfloat16), (1500, 1600, torch.float32, None), (700, 5001, torch.float16, torch.float32),
                                             (3, 8192, torch.float32, torch.float32), (40, 40000, torch.bfloat16, None)])
def test_norm_rounds_codes_once(rows, cols, xt, rt):
    """Codes are those of the 64-bit values of the 32-bit sums x + residual: all of them, also next to a tie."""
    x, w = _x(rows + cols, rows, cols, xt, 0, 1), torch.randn(cols, device="cuda")
    r = None if rt is None else _x(rows * 3 + cols, rows, cols, rt, 0, 1)
    y = L.rmsnorm(_np(x.float() if r is None else x.float() + r.float()), _np(w), float(np.float32(1e-6)))
    for fmt in FORMATS:
        codes, scales = S.sbn_quantized_empty(fmt, rows, cols)
        S.sbn_add_rmsnorm(x, w, 1e-6, residual=r, fmt=fmt, codes=codes, scales=scales)
        if fmt == S.SBN_FP8_ROW:
            top = np.abs(y).max(1)
            want, want_s = np.zeros(tuple(codes.shape), dtype=np.uint8), (top / 448).astype(np.float32)
            want[:, :cols] = L.element_codes(y * (448 / np.where(top > 0, top, 1))[:, None], L.E4M3, 128)
        else:
            want, want_s = L.quantize(y, fmt)
        assert np.array_equal(codes.cpu().numpy(), want) and np.array_equal(scales.cpu().numpy(), want_s)


def test_rows_far_apart():
    """Offsets past 32 bits: rows 3 * 2^30 bytes apart."""
    ld = 3 << 29
    buf = torch.empty(2 * ld + 4096, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((3, 999), (ld, 1))
    x.copy_(_x(5, 3, 999, torch.bfloat16))
    for fmt in FORMATS:
        codes, scales = _quantize(x, fmt)
        want_c, want_s = L.quantize(_np(x), fmt)
        assert np.array_equal(codes.cpu().numpy(), want_c) and np.array_equal(scales.cpu().numpy(), want_s)
        S.sbn_dequantize(codes, scales, fmt, x)
        assert np.array_equal(_np(x), _np(torch.from_numpy(L.values(want_c, want_s, fmt, 999)).float().bfloat16()))
    y = torch.empty(3, 999, dtype=torch.bfloat16, device="cuda")
    before = _np(x)
    S.sbn_add_rmsnorm(x, None, 1e-6, residual=x.clone(), total=x, y=y)
    assert np.array_equal(_np(x), _np(torch.from_numpy(2 * before).bfloat16()))
    want = L.rmsnorm(2 * before, None, 1e-6)
    assert np.all(np.abs(_np(y) - want) <= np.abs(want) * (NORM_REL + 2.0 ** -8 * 1.01) + 1e-37)


def test_no_rows_other_streams_and_refusals():
    codes, scales = S.sbn_quantized_empty(S.SBN_MXFP8, 0, 64)
    S.sbn_quantize(torch.empty(0, 64, device="cuda"), S.SBN_MXFP8, codes, scales)
    S.sbn_dequantize(codes, scales, S.SBN_MXFP8, torch.empty(0, 64, device="cuda"))
    S.sbn_add_rmsnorm(torch.empty(0, 64, device="cuda"), None, 1e-6, y=torch.empty(0, 64, device="cuda"))
    x = _x(9, 64, 512, torch.float32)
    want = _quantize(x, S.SBN_MXFP8)[0]
    side = torch.cuda.Stream()
    codes, scales = S.sbn_quantized_empty(S.SBN_MXFP8, 64, 512)
    side.wait_stream(torch.cuda.current_stream())
    S.sbn_quantize(x, S.SBN_MXFP8, codes, scales, stream=side)
    side.synchronize()
    assert torch.equal(codes, want)
    for bad in (lambda: S.sbn_quantize(x.double(), S.SBN_MXFP8, codes, scales), lambda: S.sbn_quantize(x.t(), S.SBN_MXFP8, codes, scales),
                lambda: S.sbn_quantize(x, 3, codes, scales), lambda: S.sbn_quantize(x, S.SBN_MXFP4, codes, scales), lambda: S.sbn_quantize(x[:5], S.SBN_MXFP8, codes, scales),
                lambda: S.sbn_quantize(x.cpu(), S.SBN_MXFP8, codes, scales), lambda: S.sbn_quantize(x[:1].expand(64, 512), S.SBN_MXFP8, codes, scales),
                lambda: S.sbn_add_rmsnorm(x, torch.ones(511, device="cuda"), 1e-6, y=torch.empty_like(x)),
                lambda: S.sbn_add_rmsnorm(x, None, 1e-6, y=torch.empty(64, 512, device="cuda", dtype=torch.bfloat16)),
                lambda: S.sbn_add_rmsnorm(x, None, 1e-6, residual=x, total=x.bfloat16())):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(S.SbnError):
        S.sbn_add_rmsnorm(x, None, 1e-6)
