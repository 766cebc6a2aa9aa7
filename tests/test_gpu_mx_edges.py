"""Edges of the microscaled operators against the float64 oracle: views, remainders, orders and sizes at which one of
their parts is used differently."""
import os
import subprocess
import sys
import threading

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


# ------------------------------------------------------------------------------------------------ a wait that runs out
# Clusters (split, and whole with more steps than stages) and pairs (one tile, and several); the first step, one of the first
# stages, one that reuses a stage, one of a second tile (steps at 4 bits; at 8 there are twice as many).
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("m,n,k,steps", [(16, 300, 4096, (0, 1)), (1, 25600, 4096, (0, 3, 9)), (100, 640, 2048, (0,)),
                                         (300, 5000, 4096, (0, 4, 11)), (2048, 4096, 4096, (0, 7, 19))])
def test_a_product_that_gives_up_waiting_returns_and_the_next_is_right(fmt, m, n, k, steps):
    """Failure detection without a fault: the wait runs out after 20 ms, the status word says so, is cleared by being
    read, and the calls after it, on the same SMs and the same tensor memory, are as before."""
    a_codes, a_scales, _ = quantized(draw(m, k, torch.float32, m + k), fmt)
    w_codes, w_scales, _ = quantized(draw(n, k, torch.float32, n + k), dq.DQ_MXFP4)
    args = (a_codes, a_scales, fmt, w_codes, w_scales, k)
    want = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
    dq.dq_mx_matmul(*args, want)
    finished()
    y = torch.empty_like(want)
    for step in (s * (1 + (fmt == dq.DQ_MXFP8)) for s in steps):
        dq.dq_mx_selftest_bounded_wait(*args, y, step, 20_000_000)
        assert dq.dq_mx_status() == dq.DQ_ERR_TIMEOUT
        finished()
        for _ in range(3):
            y.zero_()
            dq.dq_mx_matmul(*args, y)
            assert torch.equal(y, want)
        finished()
    dq.dq_mx_selftest_bounded_wait(*args, y, 1 << 40, 20_000_000)      # no CTA has that many steps: nothing runs out
    finished()
    assert torch.equal(y, want)


# ------------------------------------------------------------------------------------------------ other host threads
@pytest.mark.parametrize("m", (4, 40, 300))
def test_products_from_a_thread_that_did_nothing_else(m):
    """A host thread whose first use of the GPU is a product gives what the main thread gives."""
    n, k = 2000, 1024
    w_codes, w_scales, _ = quantized(draw(n, k, torch.float32, 1), dq.DQ_MXFP4)
    a_codes, a_scales, _ = quantized(draw(m, k, torch.float32, 2), dq.DQ_MXFP8)
    x = draw(m, k, torch.bfloat16, 3)
    work = torch.empty(dq.dq_mx_linear_workspace(dq.DQ_MXFP4, m, k), dtype=torch.uint8, device="cuda")
    y, z, other_y, other_z = (torch.zeros((m, n), dtype=torch.bfloat16, device="cuda") for _ in range(4))
    stream = torch.cuda.current_stream()
    errors = []

    def calls(y, z):
        try:
            dq.dq_mx_matmul(a_codes, a_scales, dq.DQ_MXFP8, w_codes, w_scales, k, y, stream=stream)
            dq.dq_mx_linear(x, dq.DQ_MXFP4, w_codes, w_scales, z, work, stream=stream)
        except Exception as e:
            errors.append(e)

    calls(y, z)
    thread = threading.Thread(target=calls, args=(other_y, other_z))
    thread.start()
    thread.join()
    assert not errors
    finished()
    assert torch.equal(y, other_y) and torch.equal(z, other_z) and bool(y.any()) and bool(z.any())


# ------------------------------------------------------------------------------------------------ first calls of several threads
FIRST_CALLS = """
import threading
import torch
import paper_2511_04063_b200 as dq

SHAPES = ((1, 4096, 4096), (40, 4096, 1000), (300, 4096, 2048), (100, 512, 700))
THREADS = 8
g = torch.Generator(device="cuda").manual_seed(1)
x = {s: torch.randn(s[0], s[1], device="cuda", generator=g).bfloat16() for s in SHAPES}
w = {s: (torch.randint(0, 256, (s[2], s[1] // 2), dtype=torch.uint8, device="cuda", generator=g),
         torch.full((-(-s[2] // 128) * (s[1] // 128) * 512,), 127, dtype=torch.uint8, device="cuda")) for s in SHAPES}
torch.cuda.synchronize()

def outputs(stream):
    out = []
    for fmt in (dq.DQ_MXFP8, dq.DQ_MXFP4):
        for s in SHAPES:
            y = torch.empty(s[0], s[2], dtype=torch.bfloat16, device="cuda")
            work = torch.empty(dq.dq_mx_linear_workspace(fmt, s[0], s[1]), dtype=torch.uint8, device="cuda")
            dq.dq_mx_linear(x[s], fmt, *w[s], y, work, stream=stream)
            out.append((y, work))
    stream.synchronize()
    return [y for y, _ in out]

got, errors = [None] * THREADS, []
ready = threading.Barrier(THREADS)
streams = [torch.cuda.Stream() for _ in range(THREADS)]

def first(i):
    try:
        ready.wait()
        got[i] = outputs(streams[i])
    except Exception as e:
        errors.append(repr(e))

threads = [threading.Thread(target=first, args=(i,)) for i in range(THREADS)]
for t in threads:
    t.start()
for t in threads:
    t.join()
assert not errors, errors
want = outputs(torch.cuda.current_stream())
torch.cuda.synchronize()
for ys in got:
    for y, z in zip(ys, want):
        assert torch.equal(y, z)
assert dq.dq_mx_status() == dq.DQ_OK
"""


def test_first_calls_of_several_threads():
    """A process whose first calls on the device come from eight threads at once."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    ran = subprocess.run([sys.executable, "-c", FIRST_CALLS], cwd=root, capture_output=True, text=True, timeout=300)
    assert ran.returncode == 0, ran.stderr[-3000:]


# ------------------------------------------------------------------------------------------------ weights from the call before
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("m,n,k", [(1, 4096, 2048), (17, 4096, 2048), (40, 8192, 4096), (300, 8192, 4096), (600, 1000, 1031)])
def test_linear_right_after_its_weights(fmt, m, n, k):
    """Weights that the kernel directly before dq_mx_linear writes, over others of another size of value: its product may read
    weights before its own quantisation of the tokens has ended, not before theirs."""
    w = [draw(n, k, torch.bfloat16, 1) * 4.0 ** i for i in range(4)]
    x = draw(m, k, torch.bfloat16, 2)
    codes, scales = dq.dq_mx_empty(n, k, dq.DQ_MXFP4)
    work = torch.empty(dq.dq_mx_linear_workspace(fmt, m, k), dtype=torch.uint8, device="cuda")
    want = []
    for v in w:
        dq.dq_mx_quantize(v, dq.DQ_MXFP4, codes, scales)
        torch.cuda.synchronize()
        want.append(torch.empty((m, n), dtype=torch.float32, device="cuda"))
        dq.dq_mx_linear(x, fmt, codes, scales, want[-1], work)
        torch.cuda.synchronize()
    assert not torch.equal(want[0], want[1])
    got = [torch.empty_like(y) for _ in range(8) for y in want]
    for i, y in enumerate(got):
        dq.dq_mx_quantize(w[i % 4], dq.DQ_MXFP4, codes, scales)
        dq.dq_mx_linear(x, fmt, codes, scales, y, work)
    finished()
    for i, y in enumerate(got):
        assert torch.equal(y, want[i % 4])


# ------------------------------------------------------------------------------------------------ long rows of the norm
# Relative error of y in fp32: at most 32 squares in a thread's sum, 5 additions across a warp and 5 across up to 32 warps, the
# squares' own rounding and the mean's, half of it under the root, rsqrtf good to 2 units, three products: below 2^-18.
Y_REL = 2.0 ** -18


def check_norm(x, residual, gamma, eps, fmt, codes, scales, values):
    """Scale and elements lie between those of y (1 - Y_REL) and y (1 + Y_REL)."""
    rows, k = x.shape
    _, y = mx.rmsnorm(f64(x), None if residual is None else f64(residual), None if gamma is None else f64(gamma), eps)
    c, s = codes.cpu().numpy(), mx.unpack_scales(scales.cpu().numpy(), rows, k)
    if fmt == dq.DQ_MXFP4:
        c = np.stack((c & 15, c >> 4), -1).reshape(rows, -1)
    _, lo = mx.quantize(y * (1 - Y_REL), fmt)
    _, hi = mx.quantize(y * (1 + Y_REL), fmt)
    assert ((s >= lo) & (s <= hi)).all()
    pad = np.zeros((rows, c.shape[1]))
    pad[:, :k] = np.abs(y)
    v = np.ldexp(pad.reshape(rows, -1, 32), (127 - s.astype(np.int64))[..., None]).reshape(rows, -1)
    mag = (c % mx.SIGN[fmt]).astype(np.int64)
    assert (mag >= mx.nearest_code(v * (1 - Y_REL), fmt)).all() and (mag <= mx.nearest_code(v * (1 + Y_REL), fmt)).all()
    assert torch.equal(values.cpu(), torch.from_numpy(mx.dequantize(c, s, fmt, k)).to(x.dtype))


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16, torch.float16))
@pytest.mark.parametrize("rows,k", [(3, 8195), (600, 8447), (2, 16385), (300, 16501), (3, 32767), (2, 16392), (2, 32760)])
def test_rmsnorm_of_long_rows(fmt, dtype, rows, k):
    """Four and eight pieces of 256 columns a warp: rows in whole pieces of 16 bytes, and rows that are not."""
    x, r = draw(rows, k, dtype, k), draw(rows, k, dtype, k + 1)
    gamma = (1 + 0.1 * draw(1, k, torch.float32, k + 2)[0]).to(dtype)
    codes, scales = dq.dq_mx_empty(rows, k, fmt)
    h, values = torch.empty_like(x), torch.empty_like(x)
    dq.dq_rmsnorm_quantize(x, gamma, 1e-5, fmt, codes, scales, residual=r, sum_out=h, values=values)
    check_norm(x, r, gamma, 1e-5, fmt, codes, scales, values)
    assert torch.equal(h, (x.float() + r.float()).to(dtype))
