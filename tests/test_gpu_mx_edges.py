"""Edges of the microscaled operators against the float64 oracle: views, remainders, orders and sizes at which one of
their parts is used differently."""
import numpy as np
import pytest
import torch

import paper_2511_04063_b200 as dq
from oracle import microscaling as mx

pytestmark = pytest.mark.gpu

FMTS = (dq.DQ_MXFP4, dq.DQ_MXFP8)
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # half an ulp, relative


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def draw(rows, k, dtype, seed):
    x = np.random.default_rng(seed).standard_t(3, (rows, k))
    return torch.from_numpy(x.astype(np.float32)).cuda().to(dtype)


def quantized(x, fmt):
    """(codes, scales, their values in float64): the first two on the device, from the oracle."""
    c, s = mx.quantize(f64(x), fmt)
    k = x.shape[1]
    return (torch.from_numpy(mx.pack_codes(c, fmt)).cuda(), torch.from_numpy(mx.pack_scales(s, k)).cuda(),
            mx.dequantize(c, s, fmt, k))


def check_product(y, a, w, k):
    """Products of elements and scales are exact in fp32; a sum of k of them in fp32, in steps that may truncate, is off by at
    most (k / 32 + 16) 2^-22 of the sum of magnitudes, the result is then rounded once."""
    ref = mx.product(a, w)
    bound = (k / 32 + 16) * 2.0 ** -22 * mx.product(np.abs(a), np.abs(w)) + UNIT[y.dtype] * np.abs(ref) * 1.01 + 2.0 ** -25
    assert (np.abs(f64(y) - ref) <= bound).all()


def finished():
    assert dq.dq_mx_status() == dq.DQ_OK


# ------------------------------------------------------------------------------------------------ one column
def column(rows, dtype, fill=7.0):
    """A column of every other column of a matrix: shape [rows, 1], strides that are neither 1."""
    whole = torch.full((rows, 6), fill, dtype=dtype, device="cuda")
    view = whole[:, ::2][:, 1:2]
    assert view.stride() == (6, 2)
    return whole, view


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16, torch.float16))
@pytest.mark.parametrize("rows", (2, 33, 200))
def test_one_column_of_a_matrix(fmt, dtype, rows):
    """It is read and written where it lies, and its neighbours are not."""
    _, x = column(rows, dtype)
    x.copy_(draw(rows, 1, dtype, rows))
    codes, scales, a = quantized(x, fmt)
    want = torch.from_numpy(a).to(dtype).cuda()

    def only(whole, view, value):
        assert torch.equal(view, value)
        rest = whole.clone()
        rest[:, 2:3] = 7.0
        assert bool((rest == 7.0).all())

    got_c, got_s = dq.dq_mx_empty(rows, 1, fmt)
    whole, values = column(rows, dtype)
    dq.dq_mx_quantize(x, fmt, got_c, got_s, values=values)
    assert torch.equal(got_c, codes)
    only(whole, values, want)
    whole, back = column(rows, dtype)
    dq.dq_mx_dequantize(codes, scales, fmt, back)
    only(whole, back, want)
    whole, h = column(rows, dtype)
    dq.dq_rmsnorm_quantize(x, None, 1e-5, fmt, got_c, got_s, residual=x, sum_out=h)
    only(whole, h, (x.float() * 2).to(dtype))
    # a product with one weight row writes one column
    k = 32
    t_codes, t_scales, t = quantized(draw(rows, k, torch.float32, 1), fmt)
    w_codes, w_scales, w = quantized(draw(1, k, torch.float32, 2), dq.DQ_MXFP4)
    whole, y = column(rows, dtype)
    dq.dq_mx_matmul(t_codes, t_scales, fmt, w_codes, w_scales, k, y)
    finished()
    check_product(y, t, w, k)
    only(whole, y, y.clone())
    w_codes, w_scales, w = quantized(draw(1, 1, torch.float32, 3), dq.DQ_MXFP4)
    whole, y = column(rows, dtype)
    dq.dq_mx_linear(x, fmt, w_codes, w_scales, y, torch.empty(dq.dq_mx_linear_workspace(fmt, rows, 1), dtype=torch.uint8, device="cuda"))
    finished()
    check_product(y, a, w, 1)
    only(whole, y, y.clone())


# ------------------------------------------------------------------------------------------------ a tile's last weight rows
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("k", (512, 1100, 4096))     # 2 to 32 steps: the reduction split over 2 to 8 CTAs
@pytest.mark.parametrize("m,n", [(1, 1), (1, 132), (7, 100), (16, 253), (17, 258), (40, 129), (64, 641), (100, 127), (128, 136)])
def test_split_products_at_a_weight_remainder(fmt, k, m, n):
    """The last weight rows do not fill a tile, so some threads of the cluster's sum have nothing to add; calls in a row,
    whose CTAs take over one another's shared memory, agree."""
    a_codes, a_scales, a = quantized(draw(m, k, torch.float32, m + k), fmt)
    w_codes, w_scales, w = quantized(draw(n, k, torch.float32, n + k), dq.DQ_MXFP4)
    outs = [torch.full((m, n + 3), 7.0, dtype=torch.float32, device="cuda") for _ in range(8)]
    for y in outs:
        dq.dq_mx_matmul(a_codes, a_scales, fmt, w_codes, w_scales, k, y[:, :n])
    finished()
    check_product(outs[0][:, :n], a, w, k)
    for y in outs:
        assert torch.equal(y, outs[0]) and bool((y[:, n:] == 7.0).all())
    if m <= 16:
        x = draw(m, k, torch.bfloat16, m)
        work = torch.empty(dq.dq_mx_linear_workspace(fmt, m, k), dtype=torch.uint8, device="cuda")
        y = torch.full((m, n + 3), 7.0, dtype=torch.float32, device="cuda")
        dq.dq_mx_linear(x, fmt, w_codes, w_scales, y[:, :n], work)
        finished()
        check_product(y[:, :n], mx.dequantize(*mx.quantize(f64(x), fmt), fmt, k), w, k)
        assert bool((y[:, n:] == 7.0).all())
