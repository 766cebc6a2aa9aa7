"""Parity of the microscaled operators with the float64 oracle: codes and scales bit for bit, norms and products
within bounds derived from the arithmetic, and what the entry points refuse."""
import numpy as np
import pytest
import torch

import paper_2511_04063_b200 as dq
from oracle import microscaling as mx

pytestmark = pytest.mark.gpu

FMTS = (dq.DQ_MXFP4, dq.DQ_MXFP8)
TYPES = (torch.float32, torch.bfloat16, torch.float16)
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # half an ulp, relative


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def draw(rows, k, dtype, seed, spread=0.0):
    """Heavy-tailed values on the device; `spread`: block magnitudes vary by up to 2^+-spread."""
    r = np.random.default_rng(seed)
    x = r.standard_t(3, (rows, k)) * 2.0 ** r.uniform(-spread, spread, (rows, -(-k // 32))).repeat(32, 1)[:, :k]
    return torch.from_numpy(x.astype(np.float32)).cuda().to(dtype)


def strided(t, extra, offset):
    """The same values with a row stride of k + extra, starting `offset` elements into an allocation."""
    rows, k = t.shape
    store = torch.full((rows * (k + extra) + offset,), 7.0, dtype=t.dtype, device="cuda")
    v = store[offset:offset + rows * (k + extra)].view(rows, k + extra)[:, :k]
    v.copy_(t)
    return v


def held(codes, scales, fmt, rows, k):
    """(codes, scale bytes) of the device's buffers in the oracle's order."""
    c = codes.cpu().numpy()
    if fmt == dq.DQ_MXFP4:
        c = np.stack((c & 15, c >> 4), -1).reshape(rows, -1)
    return c, mx.unpack_scales(scales.cpu().numpy(), rows, k)


def quantized(x, fmt):
    """(codes, scales, oracle values) on the device from the oracle."""
    c, s = mx.quantize(f64(x), fmt)
    k = x.shape[1]
    return (torch.from_numpy(mx.pack_codes(c, fmt)).cuda(), torch.from_numpy(mx.pack_scales(s, k)).cuda(),
            mx.dequantize(c, s, fmt, k))


def same(a, b):
    """Equal values, NaN where the other is NaN (a float16 infinity among the drawn values makes its block NaN)."""
    return a.dtype == b.dtype and torch.allclose(a.cpu(), b.cpu(), rtol=0, atol=0, equal_nan=True)


def finished():
    assert dq.dq_mx_status() == dq.DQ_OK


# ------------------------------------------------------------------------------------------------ quantise
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,k,extra,offset", [(1, 1, 0, 0), (1, 32, 0, 0), (2, 31, 0, 0), (33, 33, 3, 0), (127, 127, 0, 1),
                                                 (128, 128, 8, 0), (129, 129, 0, 0), (40, 255, 1, 1), (257, 256, 0, 8),
                                                 (1, 4096, 0, 0), (70, 1000, 24, 0), (300, 520, 0, 4), (1, 128, 0, 0), (31, 96, 0, 0), (161, 128, 0, 0),
                                                 (1000, 8, 0, 0), (97, 120, 16, 16), (1001, 103, 0, 0), (35, 100, 3, 1)])
def test_quantize_is_the_oracles_bit_for_bit(fmt, dtype, rows, k, extra, offset):
    x = strided(draw(rows, k, dtype, rows * 1000 + k, spread=9.0), extra, offset)
    codes, scales = dq.dq_mx_empty(rows, k, fmt)
    values = strided(torch.zeros_like(x), extra, offset)
    dq.dq_mx_quantize(x, fmt, codes, scales, values=values)
    c, s = held(codes, scales, fmt, rows, k)
    c_ref, s_ref = mx.quantize(f64(x), fmt)
    assert np.array_equal(s, s_ref)
    assert np.array_equal(c, c_ref)
    want = torch.from_numpy(mx.dequantize(c_ref, s_ref, fmt, k)).to(dtype)
    assert same(values, want)
    back = strided(torch.zeros_like(x), extra, offset)
    dq.dq_mx_dequantize(codes, scales, fmt, back)
    assert same(back, want)
    if extra:      # the gaps between the rows are not written
        whole = torch.as_strided(back, (rows, k + extra), (k + extra, 1), back.storage_offset())
        assert bool((whole[:, k:] == 7.0).all())


@pytest.mark.parametrize("fmt", FMTS)
def test_quantize_special_values(fmt):
    x = torch.zeros((6, 160), dtype=torch.float32)
    x[0, 3] = float("nan"); x[0, 64] = 1.0
    x[1, 33] = float("inf"); x[1, 0] = -2.5
    x[2, 10] = 2.0 ** -149; x[2, 40] = -(2.0 ** -126); x[2, 70] = 2.0 ** -127
    x[3, 0] = 3.4028234e38; x[3, 31] = -1e30; x[3, 32] = 2.0 ** 127
    x[4] = -0.0
    x[5, :32] = torch.arange(32) * 0.25
    codes, scales = dq.dq_mx_empty(6, 160, fmt)
    values = torch.empty_like(x, device="cuda")
    dq.dq_mx_quantize(x.cuda(), fmt, codes, scales, values=values)
    c, s = held(codes, scales, fmt, 6, 160)
    c_ref, s_ref = mx.quantize(f64(x), fmt)
    assert np.array_equal(s, s_ref) and np.array_equal(c, c_ref)
    want = mx.dequantize(c_ref, s_ref, fmt, 160)
    got = f64(values)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~np.isnan(want)], want[~np.isnan(want)])


def test_quantize_in_place_empty_and_on_another_stream():
    x = draw(200, 640, torch.bfloat16, 3)
    codes, scales = dq.dq_mx_empty(200, 640, dq.DQ_MXFP8)
    want = torch.empty_like(x)
    dq.dq_mx_quantize(x, dq.DQ_MXFP8, codes, scales, values=want)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    again = x.clone()
    c2, s2 = dq.dq_mx_empty(200, 640, dq.DQ_MXFP8)
    torch.cuda.synchronize()
    dq.dq_mx_quantize(again, dq.DQ_MXFP8, c2, s2, values=again, stream=s)
    s.synchronize()
    assert torch.equal(again, want) and torch.equal(codes, c2)
    none = torch.empty((0, 64), dtype=torch.float32, device="cuda")
    dq.dq_mx_quantize(none, dq.DQ_MXFP4, *dq.dq_mx_empty(0, 64, dq.DQ_MXFP4))


def test_offsets_past_32_bits():
    """2.4e9 values: byte and element offsets of the last rows need 64 bits."""
    rows, k = 75000, 32000
    x = torch.zeros((rows, k), dtype=torch.bfloat16, device="cuda")
    tail = draw(200, k, torch.bfloat16, 8)
    x[-200:] = tail
    codes, scales = dq.dq_mx_empty(rows, k, dq.DQ_MXFP8)
    dq.dq_rmsnorm_quantize(x, None, 1e-5, dq.DQ_MXFP8, codes, scales)
    few_c, few_s = dq.dq_mx_empty(200, k, dq.DQ_MXFP8)
    dq.dq_rmsnorm_quantize(tail.contiguous(), None, 1e-5, dq.DQ_MXFP8, few_c, few_s)
    assert torch.equal(codes[-200:], few_c)
    dq.dq_mx_quantize(x, dq.DQ_MXFP8, codes, scales)
    dq.dq_mx_quantize(tail.contiguous(), dq.DQ_MXFP8, few_c, few_s)
    assert torch.equal(codes[-200:], few_c)
    dq.dq_mx_dequantize(codes, scales, dq.DQ_MXFP8, x)
    dq.dq_mx_dequantize(few_c, few_s, dq.DQ_MXFP8, tail)
    assert torch.equal(x[-200:], tail) and not bool(x[:-200].any())


# ------------------------------------------------------------------------------------------------ norm
# Relative error of y in fp32: the sum of squares has non-negative terms and at most 110 roundings in a chain (32 in a
# thread, 5 across a warp, 32 warps, the squares' own and the mean's), the square root halves it, rsqrtf is good to 2 units, and
# three products follow: (110 / 2 + 2 * 2 + 3) * 2^-24 < 2^-18.
Y_REL = 2.0 ** -18


def check_norm(x, residual, gamma, eps, fmt, codes, scales, sum_out, values):
    rows, k = x.shape
    h, y = mx.rmsnorm(f64(x), None if residual is None else f64(residual), None if gamma is None else f64(gamma), eps)
    if sum_out is not None:     # one rounding to fp32, one to the type
        assert (np.abs(f64(sum_out) - h) <= (UNIT[x.dtype] + 2.0 ** -24) * np.abs(h) * 1.001 + 2.0 ** -25).all()
    c, s = held(codes, scales, fmt, rows, k)
    _, s_lo = mx.quantize(y * (1 - Y_REL), fmt)
    _, s_hi = mx.quantize(y * (1 + Y_REL), fmt)
    assert ((s >= s_lo) & (s <= s_hi)).all()
    got = mx.dequantize(c, s, fmt, k)
    # with the kernel's scale every element lies between those of y's two bounds
    pad = np.zeros((rows, c.shape[1]))
    pad[:, :k] = np.abs(y)
    v = np.ldexp(pad.reshape(rows, -1, 32), (127 - s.astype(np.int64))[..., None]).reshape(rows, -1)
    mag = (c % mx.SIGN[fmt]).astype(np.int64)
    assert (mag >= mx.nearest_code(v * (1 - Y_REL), fmt)).all() and (mag <= mx.nearest_code(v * (1 + Y_REL), fmt)).all()
    assert (np.signbit(got) == np.signbit(y))[got != 0].all()
    if values is not None:
        assert torch.equal(values.cpu(), torch.from_numpy(got).to(x.dtype))


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,k,extra,offset", [(1, 1, 0, 0), (3, 31, 0, 0), (5, 128, 0, 0), (9, 130, 6, 2), (2, 513, 0, 0), (130, 512, 0, 0),
                                                 (4, 1000, 8, 8), (2, 4096, 0, 0), (3, 5120, 0, 0), (2, 8200, 0, 0), (1, 32768, 0, 0), (1, 96, 0, 0),
                                                 (33, 128, 0, 0), (100, 8, 8, 8), (101, 103, 0, 0), (19, 127, 1, 1)])
def test_rmsnorm_quantize(fmt, dtype, rows, k, extra, offset):
    x = strided(draw(rows, k, dtype, k), extra, offset)
    residual = strided(draw(rows, k, dtype, k + 1), extra, offset)
    for g_type in (None, torch.float32, dtype):
        gamma = None if g_type is None else (1 + 0.1 * draw(1, k, torch.float32, k + 2)[0]).to(g_type)
        for r in (None, residual):
            codes, scales = dq.dq_mx_empty(rows, k, fmt)
            h, values = strided(torch.zeros_like(x), extra, offset), strided(torch.zeros_like(x), extra, offset)
            dq.dq_rmsnorm_quantize(x, gamma, 1e-5, fmt, codes, scales, residual=r, sum_out=h, values=values)
            check_norm(x, r, gamma, 1e-5, fmt, codes, scales, h, values)


def test_rmsnorm_in_place_and_bare():
    x, r = draw(50, 1024, torch.bfloat16, 5), draw(50, 1024, torch.bfloat16, 6)
    c1, s1 = dq.dq_mx_empty(50, 1024, dq.DQ_MXFP8)
    dq.dq_rmsnorm_quantize(x, None, 1e-6, dq.DQ_MXFP8, c1, s1, residual=r)     # no sum, no values
    check_norm(x, r, None, 1e-6, dq.DQ_MXFP8, c1, s1, None, None)
    for target in ("x", "residual"):
        a, b = x.clone(), r.clone()
        c2, s2 = dq.dq_mx_empty(50, 1024, dq.DQ_MXFP8)
        dq.dq_rmsnorm_quantize(a, None, 1e-6, dq.DQ_MXFP8, c2, s2, residual=b, sum_out=a if target == "x" else b)
        assert torch.equal(c1, c2)
        assert torch.equal(a if target == "x" else b, (x.float() + r.float()).to(torch.bfloat16))


@pytest.mark.parametrize("rows,k", [(2000, 700), (10000, 512), (1500, 4096), (700, 4099)])
def test_rmsnorm_many_rows(rows, k):
    """The variants for many rows: several pieces a warp, several rows a CTA, rows that are not in whole pieces."""
    x, r = draw(rows, k, torch.bfloat16, 1), draw(rows, k, torch.bfloat16, 2)
    gamma = (1 + 0.1 * draw(1, k, torch.float32, 3)[0]).to(torch.bfloat16)
    codes, scales = dq.dq_mx_empty(rows, k, dq.DQ_MXFP8)
    h, values = torch.empty_like(x), torch.empty_like(x)
    dq.dq_rmsnorm_quantize(x, gamma, 1e-5, dq.DQ_MXFP8, codes, scales, residual=r, sum_out=h, values=values)
    check_norm(x, r, gamma, 1e-5, dq.DQ_MXFP8, codes, scales, h, values)


def test_rmsnorm_rows_are_independent():
    """A row with a NaN, one with an infinity and one of zeros beside ordinary ones."""
    x = draw(8, 256, torch.float32, 4)
    clean = x.clone()
    x[2, 17] = float("nan")
    x[4, 200] = float("inf")
    x[6] = 0.0
    out = []
    for t in (x, clean):
        codes, scales = dq.dq_mx_empty(8, 256, dq.DQ_MXFP8)
        values = torch.empty_like(t)
        dq.dq_rmsnorm_quantize(t, None, 1e-5, dq.DQ_MXFP8, codes, scales, values=values)
        out.append(values.cpu())
    for r in (0, 1, 3, 5, 7):
        assert torch.equal(out[0][r], out[1][r])
    assert bool(torch.isnan(out[0][2]).all())
    assert bool(torch.isnan(out[0][4, 192:224]).all())           # infinity / infinity in its block, 0 elsewhere
    assert bool((out[0][4, :192] == 0).all()) and bool((out[0][4, 224:] == 0).all())
    assert bool((out[0][6] == 0).all())


# ------------------------------------------------------------------------------------------------ product
def check_product(y, a, w, k):
    """Products of elements and scales are exact in fp32; a sum of k of them in fp32, in steps that may truncate, is off by at
    most (k / 32 + 16) 2^-22 of the sum of magnitudes, the result is then rounded once."""
    ref = mx.product(a, w)
    bound = (k / 32 + 16) * 2.0 ** -22 * mx.product(np.abs(a), np.abs(w)) + UNIT[y.dtype] * np.abs(ref) * 1.01 + 2.0 ** -25
    got = f64(y)
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    fine = np.isfinite(ref)
    assert (np.abs(got - ref)[fine] <= bound[fine]).all()


SHAPES = [(1, 1, 1), (1, 128, 32), (3, 5, 31), (16, 128, 128), (17, 130, 129), (7, 300, 1000), (32, 64, 257), (33, 257, 384),
          (64, 1, 2048), (65, 384, 300), (128, 256, 512), (129, 200, 640), (200, 1000, 100), (256, 512, 1152), (300, 333, 777),
          (300, 1, 256), (257, 8, 31), (70, 129, 4096)]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_matmul(fmt, m, n, k):
    a_codes, a_scales, a = quantized(draw(m, k, torch.float32, m + k), fmt)
    w_codes, w_scales, w = quantized(draw(n, k, torch.float32, n + k), dq.DQ_MXFP4)
    for dtype, extra, offset in ((torch.bfloat16, 0, 0), (torch.float16, 3, 1), (torch.float32, 0, 0), (torch.float32, 4, 4)):
        y = strided(torch.full((m, n), float("nan"), dtype=dtype, device="cuda"), extra, offset)
        dq.dq_mx_matmul(a_codes, a_scales, fmt, w_codes, w_scales, k, y)
        finished()
        check_product(y, a, w, k)
        if extra:
            whole = torch.as_strided(y, (m, n + extra), (n + extra, 1), y.storage_offset())
            assert bool((whole[:, n:] == 7.0).all())


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("m,n,k", [(1, 2048, 2048), (5, 1000, 4096), (100, 4096, 640), (513, 1029, 1031), (2048, 1280, 512),
                                   (1000, 2568, 2560)])
def test_matmul_larger(fmt, m, n, k):
    a_codes, a_scales, a = quantized(draw(m, k, torch.float32, m + k), fmt)
    w_codes, w_scales, w = quantized(draw(n, k, torch.float32, n + k), dq.DQ_MXFP4)
    y = torch.full((m, n), float("nan"), dtype=torch.float32, device="cuda")
    dq.dq_mx_matmul(a_codes, a_scales, fmt, w_codes, w_scales, k, y)
    finished()
    check_product(y, a, w, k)
    again = torch.empty_like(y)
    dq.dq_mx_matmul(a_codes, a_scales, fmt, w_codes, w_scales, k, again)
    assert torch.equal(y, again)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("m", [4, 150, 700])
def test_matmul_keeps_rows_apart(fmt, m):
    """A NaN block in one token and one weight row reaches that row and column of the result only; undefined scales of rows
    past the last one reach nothing."""
    n, k = 260, 544
    x, wt = draw(m, k, torch.float32, 1), draw(n, k, torch.float32, 2)
    a_codes, a_scales, a = quantized(x, fmt)
    w_codes, w_scales, w = quantized(wt, dq.DQ_MXFP4)
    r, b = np.meshgrid(np.arange(-(-m // 128) * 128), np.arange(-(-k // 128) * 4), indexing="ij")
    a_scales[torch.from_numpy(mx.scale_index(r, b, k)[m:].ravel()).cuda()] = 255
    r, b = np.meshgrid(np.arange(-(-n // 128) * 128), np.arange(-(-k // 128) * 4), indexing="ij")
    w_scales[torch.from_numpy(mx.scale_index(r, b, k)[n:].ravel()).cuda()] = 255
    a_scales[int(mx.scale_index(m - 1, 16, k))] = 255
    w_scales[int(mx.scale_index(7, 0, k))] = 255
    y = torch.zeros((m, n), dtype=torch.float32, device="cuda")
    dq.dq_mx_matmul(a_codes, a_scales, fmt, w_codes, w_scales, k, y)
    finished()
    bad = torch.isnan(y).cpu()
    want = torch.zeros((m, n), dtype=torch.bool)
    want[m - 1] = True
    want[:, 7] = True
    assert torch.equal(bad, want)
    keep = [i for i in range(n) if i != 7]
    if m > 1:
        check_product(y[:m - 1, keep], a[:m - 1], w[keep], k)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("m,n,k", [(3, 256, 33000), (64, 40000, 160), (130, 20000, 384), (1200, 4100, 96)])
def test_matmul_many_steps_and_many_tiles(fmt, m, n, k):
    """More pipeline steps than stages by far; more tiles than SMs; the token tile's and the weight tile's last rows."""
    a_codes, a_scales, a = quantized(draw(m, k, torch.float32, 1), fmt)
    w_codes, w_scales, w = quantized(draw(n, k, torch.float32, 2), dq.DQ_MXFP4)
    y = torch.full((m, n), float("nan"), dtype=torch.float32, device="cuda")
    dq.dq_mx_matmul(a_codes, a_scales, fmt, w_codes, w_scales, k, y)
    finished()
    check_product(y, a, w, k)


@pytest.mark.parametrize("fmt", FMTS)
def test_scales_reach_the_ends_of_fp32(fmt):
    """Products of the largest and smallest scales: 2^100 * 2^-100 is ordinary."""
    x = draw(20, 256, torch.float32, 1)
    w = draw(40, 256, torch.float32, 2)
    a_codes, a_scales, a = quantized(x * 2.0 ** 100, fmt)
    w_codes, w_scales, wv = quantized(w * 2.0 ** -100, dq.DQ_MXFP4)
    y = torch.empty((20, 40), dtype=torch.float32, device="cuda")
    dq.dq_mx_matmul(a_codes, a_scales, fmt, w_codes, w_scales, 256, y)
    check_product(y, a, wv, 256)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", [(1, 300, 1000), (2, 2048, 4096), (9, 130, 257), (16, 640, 8192), (17, 128, 100), (150, 257, 640), (600, 700, 520)])
def test_linear_is_quantize_then_matmul(fmt, dtype, m, n, k):
    x = strided(draw(m, k, dtype, m + n), 5 if k % 2 else 8, 1 if k % 2 else 0)
    w_codes, w_scales, w = quantized(draw(n, k, torch.float32, n), dq.DQ_MXFP4)
    y = torch.full((m, n), float("nan"), dtype=torch.float32, device="cuda")
    work = torch.empty(dq.dq_mx_linear_workspace(fmt, m, k), dtype=torch.uint8, device="cuda")
    dq.dq_mx_linear(x, fmt, w_codes, w_scales, y, work)
    finished()
    a = mx.dequantize(*mx.quantize(f64(x), fmt), fmt, k)
    check_product(y, a, w, k)
    half = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
    dq.dq_mx_linear(x, fmt, w_codes, w_scales, half, work)
    assert torch.equal(half, y.to(torch.bfloat16))


def test_linear_passes_non_finite_tokens_on():
    for m in (3, 40, 300):
        x = draw(m, 512, torch.bfloat16, m)
        x[1, 100] = float("inf")
        w_codes, w_scales, _ = quantized(draw(200, 512, torch.float32, 9), dq.DQ_MXFP4)
        y = torch.empty((m, 200), dtype=torch.bfloat16, device="cuda")
        work = torch.empty(dq.dq_mx_linear_workspace(dq.DQ_MXFP4, m, 512), dtype=torch.uint8, device="cuda")
        dq.dq_mx_linear(x, dq.DQ_MXFP4, w_codes, w_scales, y, work)
        bad = torch.isnan(y)
        assert bool(bad[1].all()) and int(bad.sum()) == 200


def test_calls_in_a_graph_and_in_a_row():
    """The chain of a layer captured and replayed on new inputs; consecutive calls share one workspace."""
    m, k, n = 24, 1024, 768
    w_codes, w_scales, w = quantized(draw(n, k, torch.float32, 1), dq.DQ_MXFP4)
    x, r = draw(m, k, torch.bfloat16, 2), draw(m, k, torch.bfloat16, 3)
    codes, scales = dq.dq_mx_empty(m, k, dq.DQ_MXFP8)
    y, z = torch.empty((m, n), dtype=torch.bfloat16, device="cuda"), torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
    work = torch.empty(dq.dq_mx_linear_workspace(dq.DQ_MXFP4, m, k), dtype=torch.uint8, device="cuda")

    def chain():
        dq.dq_rmsnorm_quantize(x, None, 1e-5, dq.DQ_MXFP8, codes, scales, residual=r, sum_out=r)
        dq.dq_mx_matmul(codes, scales, dq.DQ_MXFP8, w_codes, w_scales, k, y)
        dq.dq_mx_linear(r, dq.DQ_MXFP4, w_codes, w_scales, z, work)
        dq.dq_mx_linear(x, dq.DQ_MXFP4, w_codes, w_scales, z, work)

    keep = r.clone()
    chain()
    torch.cuda.synchronize()
    r.copy_(keep)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        chain()
    x2 = draw(m, k, torch.bfloat16, 4)
    x.copy_(x2)
    r.copy_(keep)
    g.replay()
    torch.cuda.synchronize()
    got_y, got_z, got_r = y.clone(), z.clone(), r.clone()
    r.copy_(keep)
    chain()
    torch.cuda.synchronize()
    assert torch.equal(got_y, y) and torch.equal(got_z, z) and torch.equal(got_r, r)
    a = mx.dequantize(*mx.quantize(f64(x2), dq.DQ_MXFP4), dq.DQ_MXFP4, k)
    check_product(z, a, w, k)


def test_two_streams_at_once():
    """The same chain on two streams with buffers of their own: the results are those of one stream alone."""
    m, k, n = 8, 2048, 1536
    w = quantized(draw(n, k, torch.float32, 1), dq.DQ_MXFP4)[:2]
    sets = []
    for seed in (2, 3):
        x = draw(m, k, torch.bfloat16, seed)
        sets.append((x, *dq.dq_mx_empty(m, k, dq.DQ_MXFP8), torch.empty((m, n), dtype=torch.bfloat16, device="cuda"),
                     torch.empty((m, n), dtype=torch.bfloat16, device="cuda"),
                     torch.empty(dq.dq_mx_linear_workspace(dq.DQ_MXFP4, m, k), dtype=torch.uint8, device="cuda")))

    def chain(s, stream=None):
        x, codes, scales, y, z, work = s
        dq.dq_rmsnorm_quantize(x, None, 1e-5, dq.DQ_MXFP8, codes, scales, stream=stream)
        dq.dq_mx_matmul(codes, scales, dq.DQ_MXFP8, *w, k, y, stream=stream)
        dq.dq_mx_linear(x, dq.DQ_MXFP4, *w, z, work, stream=stream)

    want = []
    for s in sets:
        chain(s)
        want.append((s[3].clone(), s[4].clone()))
    torch.cuda.synchronize()
    for s in sets:
        s[3].zero_()
        s[4].zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        for s, stream in zip(sets, streams):
            chain(s, stream)
    torch.cuda.synchronize()
    finished()
    for s, (y, z) in zip(sets, want):
        assert torch.equal(s[3], y) and torch.equal(s[4], z)


# ------------------------------------------------------------------------------------------------ refusals
def test_refusals():
    x = draw(4, 64, torch.bfloat16, 1)
    codes, scales = dq.dq_mx_empty(4, 64, dq.DQ_MXFP4)
    y = torch.empty((4, 4), dtype=torch.bfloat16, device="cuda")
    for call in (lambda: dq.dq_mx_quantize(x, 2, codes, scales),
                 lambda: dq.dq_mx_quantize(x.cpu(), dq.DQ_MXFP4, codes, scales),
                 lambda: dq.dq_mx_quantize(x.double(), dq.DQ_MXFP4, codes, scales),
                 lambda: dq.dq_mx_quantize(x[0], dq.DQ_MXFP4, codes, scales),
                 lambda: dq.dq_mx_quantize(x.t(), dq.DQ_MXFP4, codes, scales),
                 lambda: dq.dq_mx_quantize(x, dq.DQ_MXFP8, codes, scales),                # codes too small for 8 bits
                 lambda: dq.dq_mx_quantize(x, dq.DQ_MXFP4, codes, scales[:-1]),
                 lambda: dq.dq_mx_quantize(x, dq.DQ_MXFP4, codes, scales, values=x.float()),
                 lambda: dq.dq_mx_quantize(x, dq.DQ_MXFP4, codes, scales, values=x[:3]),
                 lambda: dq.dq_rmsnorm_quantize(x, torch.ones(63, device="cuda"), 1e-5, dq.DQ_MXFP4, codes, scales),
                 lambda: dq.dq_rmsnorm_quantize(x, None, 1e-5, dq.DQ_MXFP4, codes, scales, residual=x.float()),
                 lambda: dq.dq_mx_matmul(codes, scales, dq.DQ_MXFP4, codes, scales, 300, y),
                 lambda: dq.dq_mx_matmul(*dq.dq_mx_empty(4, 256, dq.DQ_MXFP4), dq.DQ_MXFP4, *dq.dq_mx_empty(4, 256, dq.DQ_MXFP4), 64, y),
                 lambda: dq.dq_mx_linear(x, dq.DQ_MXFP4, codes, scales, y, scales[:8])):
        with pytest.raises(ValueError):
            call()
    for call, status in ((lambda: dq.dq_rmsnorm_quantize(x, None, -1.0, dq.DQ_MXFP4, codes, scales), dq.DQ_ERR_INVALID_ARG),
                         (lambda: dq.dq_mx_quantize(x, dq.DQ_MXFP4, torch.empty(1000, dtype=torch.uint8, device="cuda")[1:],
                                                    scales), dq.DQ_ERR_UNSUPPORTED)):
        with pytest.raises(dq.DartQuantError) as e:
            call()
        assert e.value.status == status
    wide = torch.zeros((1, 33000), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(dq.DartQuantError) as e:
        dq.dq_rmsnorm_quantize(wide, None, 1e-5, dq.DQ_MXFP4, *dq.dq_mx_empty(1, 33000, dq.DQ_MXFP4))
    assert e.value.status == dq.DQ_ERR_UNSUPPORTED
    finished()
