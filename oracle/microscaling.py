"""Float64 oracle of the microscaled operators: OCP microscaling blocks (32 values, E8M0 scale, E2M1 or E4M3 elements),
the root-mean-square norm in front of them and the product of quantised operands.  Elements are found by comparing with
every value of the type; the layout is written out index by index."""
import numpy as np

MXFP4, MXFP8 = 0, 1
EMAX = {MXFP4: 2, MXFP8: 8}
BLOCK = 32

# Non-negative values of the element types by their code (sign bit clear).
E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=np.float64)
E4M3 = np.array([(m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127],
                dtype=np.float64)
GRID = {MXFP4: E2M1, MXFP8: E4M3}
SIGN = {MXFP4: 8, MXFP8: 128}


def nearest_code(v, fmt):
    """Code of the element nearest to v (ties to the even code, saturating), sign included."""
    g = GRID[fmt]
    a = np.abs(v)
    hi = np.clip(np.searchsorted(g, a, side="left"), 1, len(g) - 1)   # g[hi - 1] < a <= g[hi]
    lo = hi - 1
    below, above = a - g[lo], g[hi] - a
    code = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    return code + np.where(np.signbit(v), SIGN[fmt], 0)


def code_value(code, fmt):
    mag = code % SIGN[fmt]
    if fmt == MXFP8 and np.any(mag == 127):
        raise ValueError("the NaN element is never written")
    return GRID[fmt][mag] * np.where(code >= SIGN[fmt], -1.0, 1.0)


def quantize(x, fmt):
    """(codes [rows][128 * tiles], scale bytes [rows][4 * tiles]) of x [rows][k]."""
    x = np.asarray(x, dtype=np.float64)
    rows, k = x.shape
    tiles = -(-k // 128)
    xp = np.zeros((rows, tiles * 128))
    xp[:, :k] = x
    b = xp.reshape(rows, -1, BLOCK)
    bad = ~np.isfinite(b).all(axis=2)
    amax = np.where(bad, 1.0, np.abs(np.where(bad[..., None], 0, b)).max(axis=2))
    e = np.where(amax > 0, np.frexp(np.where(amax > 0, amax, 1.0))[1] - 1 - EMAX[fmt], -127)
    s = np.clip(e, -127, 127) + 127
    v = np.ldexp(np.where(bad[..., None], 0.0, b), -(s[..., None] - 127))
    codes = nearest_code(v, fmt)
    return codes.reshape(rows, -1).astype(np.uint8), np.where(bad, 255, s).astype(np.uint8)


def dequantize(codes, scales, fmt, k):
    v = code_value(codes.astype(np.int64), fmt).reshape(codes.shape[0], -1, BLOCK)
    s = scales.astype(np.int64)
    out = np.ldexp(v, (s - 127)[..., None])
    return np.where((s == 255)[..., None], np.nan, out).reshape(codes.shape[0], -1)[:, :k]


def pack_codes(codes, fmt):
    """Codes as bytes: two 4-bit codes a byte, the even one low."""
    if fmt == MXFP8:
        return codes
    return (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8)


def scale_index(row, block, k):
    return ((row // 128) * (-(-k // 128)) + block // 4) * 512 + row % 32 * 16 + row // 32 % 4 * 4 + block % 4


def pack_scales(scales, k):
    """Scale bytes in tile order; bytes of rows past the last are 0 here and undefined in the library."""
    rows, blocks = scales.shape
    out = np.zeros(-(-rows // 128) * (-(-k // 128)) * 512, dtype=np.uint8)
    r, b = np.meshgrid(np.arange(rows), np.arange(blocks), indexing="ij")
    out[scale_index(r, b, k)] = scales
    return out


def unpack_scales(tiles, rows, k):
    r, b = np.meshgrid(np.arange(rows), np.arange(-(-k // 128) * 4), indexing="ij")
    return tiles[scale_index(r, b, k)]


def rmsnorm(x, residual, gamma, eps):
    """(h, y)"""
    h = np.asarray(x, dtype=np.float64)
    if residual is not None:
        h = h + residual
    y = h / np.sqrt((h * h).mean(axis=1, keepdims=True) + eps)
    return h, y if gamma is None else y * gamma


def product(a_values, w_values):
    return a_values @ w_values.T
