"""Pins of the microscaling oracle: the types' tables, closed forms of a block, error bounds and the layout."""
import numpy as np
import pytest

from oracle import microscaling as mx

FMTS = (mx.MXFP4, mx.MXFP8)


def test_element_tables():
    assert mx.E2M1.max() == 6 and len(mx.E2M1) == 8
    assert mx.E4M3.max() == 448 and mx.E4M3[1] == 2.0 ** -9 and mx.E4M3[8] == 2.0 ** -6 and mx.E4M3[0x38] == 1.0
    for g in mx.GRID.values():
        assert (np.diff(g) > 0).all()


@pytest.mark.parametrize("fmt", FMTS)
def test_every_element_is_its_own_code_and_ties_go_to_even(fmt):
    g = mx.GRID[fmt]
    assert np.array_equal(mx.nearest_code(g, fmt), np.arange(len(g)))
    assert np.array_equal(mx.nearest_code(-g[1:], fmt), np.arange(1, len(g)) + mx.SIGN[fmt])
    mids = (g[1:] + g[:-1]) / 2
    code = mx.nearest_code(mids, fmt)
    assert (code % 2 == 0).all() and (np.abs(code - np.arange(len(mids)) - 0.5) == 0.5).all()
    assert mx.nearest_code(np.array([1e9]), fmt)[0] == len(g) - 1


def test_hand_worked_block():
    x = np.zeros((1, 32))
    x[0, :6] = [7.9, -3.6, 5.0, 2.5, 0.25, -0.26]     # largest exponent 2, so the scale is 2^0
    codes, scales = mx.quantize(x, mx.MXFP4)
    assert scales[0, 0] == 127
    assert mx.dequantize(codes, scales, mx.MXFP4, 6).tolist() == [[6, -4, 4, 2, 0, -0.5]]
    x *= 2.0 ** -40
    codes2, scales2 = mx.quantize(x, mx.MXFP4)
    assert scales2[0, 0] == 87 and np.array_equal(codes, codes2)


@pytest.mark.parametrize("fmt,bits", [(mx.MXFP4, 1), (mx.MXFP8, 3)])
def test_error_of_a_block_is_half_a_step_or_the_saturation(fmt, bits):
    x = np.random.default_rng(0).standard_t(3, (64, 300))
    y = mx.dequantize(*mx.quantize(x, fmt), fmt, 300)
    full = np.zeros((64, 320))
    full[:, :300] = np.abs(x)
    amax = full.reshape(64, -1, 32).max(2).repeat(32, 1)[:, :300]
    scale = 2.0 ** (np.floor(np.log2(amax)) - mx.EMAX[fmt])
    top = mx.GRID[fmt][-1] * scale
    emin = 0 if fmt == mx.MXFP4 else -6
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.abs(x) / scale)), emin) - bits) * scale
    assert (np.abs(y - np.clip(x, -top, top)) <= step / 2).all()
    assert (np.abs(x - np.clip(x, -top, top)) <= amax / 4 + 1e-12).all()


@pytest.mark.parametrize("fmt", FMTS)
def test_non_finite_zero_and_tiny_blocks(fmt):
    x = np.zeros((4, 96))
    x[0, 5] = np.nan
    x[1, 40] = -np.inf
    x[2, 70] = 2.0 ** -149
    codes, scales = mx.quantize(x, fmt)
    assert (scales[0, :4] == [255, 0, 0, 0]).all() and (scales[1, :4] == [0, 255, 0, 0]).all() and (scales[2:] == 0).all()
    y = mx.dequantize(codes, scales, fmt, 96)
    assert np.isnan(y[0, :32]).all() and np.isnan(y[1, 32:64]).all() and (y[2:] == 0).all() and (y[0, 32:] == 0).all()


def test_scale_tiles_hold_every_scale_once():
    rows, k = 300, 1000
    r, b = np.meshgrid(np.arange(384), np.arange(32), indexing="ij")
    assert np.array_equal(np.sort(mx.scale_index(r, b, k).ravel()), np.arange(3 * 8 * 512))
    s = np.random.default_rng(1).integers(0, 255, (rows, 32)).astype(np.uint8)
    assert np.array_equal(mx.unpack_scales(mx.pack_scales(s, k), rows, k), s)


def test_norm_closed_forms():
    x = np.array([[3.0, 4.0]])
    h, y = mx.rmsnorm(x, None, None, 0.0)
    assert np.allclose(y, x / np.sqrt(12.5)) and np.array_equal(h, x)
    h, y2 = mx.rmsnorm(x, x, np.array([1.0, 2.0]), 0.0)
    assert np.array_equal(h, 2 * x) and np.allclose(y2, y * [1, 2])
