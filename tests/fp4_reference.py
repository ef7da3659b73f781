"""Plain forms of the 4-bit operands with block scales, for the tests (numpy; shares no code with the library): the packed layout, the quantiser's
definition, products in 64 bits."""
from __future__ import annotations

import numpy as np
import torch

from fp8_reference import SMALLEST, UNIT, f64  # noqa: F401

BLOCK = {"nvfp4": 16, "mxfp4": 32}
MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E4M3 = np.array([(m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)) for e in range(16) for m in range(8)])
E4M3[127] = np.nan


def blocks(n, fmt):
    return -(-n // BLOCK[fmt])


def bytes_of(t) -> np.ndarray:
    return t.detach().cpu().numpy()


def codes(q, cols) -> np.ndarray:
    """(..., R, ceil(C / 2)) bytes as (..., R, C) codes, the first of a pair in the low half."""
    b = bytes_of(q)
    return np.stack([b & 15, b >> 4], -1).reshape(*b.shape[:-1], -1)[..., :cols]


def decode(code) -> np.ndarray:
    return np.where(code & 8, -1.0, 1.0) * MAGNITUDES[code & 7]


def scale_bytes(tiles, rows, cols, fmt) -> np.ndarray:
    """The scale of row r, block b: byte 16 (r % 32) + 4 (r % 128 / 32) + b % 4 of tile (r / 128, b / 4)."""
    t = bytes_of(tiles)
    r, b = np.arange(rows)[:, None], np.arange(blocks(cols, fmt))[None, :]
    return t[..., r // 128, b // 4, 16 * (r % 32) + 4 * (r % 128 // 32) + b % 4]


def scale_values(b, fmt) -> np.ndarray:
    return E4M3[b & 127] if fmt == "nvfp4" else np.where(b == 255, np.nan, 2.0 ** (b.astype(np.float64) - 127))


def tiles_from(b, fmt) -> np.ndarray:
    """Scale tiles of a matrix of scale bytes; zeros where it has none."""
    R, B = b.shape[-2:]
    out = np.zeros((*b.shape[:-2], -(-R // 128), -(-B // 4), 512), np.uint8)
    r, c = np.arange(R)[:, None], np.arange(B)[None, :]
    out[..., r // 128, c // 4, 16 * (r % 32) + 4 * (r % 128 // 32) + c % 4] = b
    return out


def pack(code) -> np.ndarray:
    C = code.shape[-1]
    wide = np.concatenate([code, np.zeros((*code.shape[:-1], C & 1), code.dtype)], -1).astype(np.uint8)
    return wide[..., 0::2] | (wide[..., 1::2] << 4)


def spread(s, fmt, cols) -> np.ndarray:
    return np.repeat(s, BLOCK[fmt], -1)[..., :cols]


def values(q, tiles, cols, fmt, factor=1.0, places=None) -> np.ndarray:
    """What a copy stands for, in 64 bits; places: the scale row of each row (laid out per group)."""
    c = codes(q, cols)
    rows = c.shape[-2]
    if places is None:
        s = scale_values(scale_bytes(tiles, rows, cols, fmt), fmt)
    else:
        s = scale_values(scale_bytes(tiles, tiles.shape[-3] * 128, cols, fmt), fmt)[places]
    return decode(c) * spread(s, fmt, cols) * np.asarray(factor, np.float64).reshape(-1, 1, 1)[0 if c.ndim == 2 else slice(None)]


def nearest_code(v) -> np.ndarray:
    """Codes of the nearest magnitudes of v, ties to the even code; the sign of v."""
    m = np.abs(v)
    mid = (MAGNITUDES[1:] + MAGNITUDES[:-1]) / 2
    up = np.array([i % 2 == 1 for i in range(7)])            # the tie between codes i and i + 1 goes up where i is odd
    code = np.zeros(v.shape, np.uint8)
    for i in range(7):
        code += ((m > mid[i]) | ((m == mid[i]) & up[i])).astype(np.uint8)
    return code | (np.signbit(v).astype(np.uint8) << 3)


def nearest_e4m3(u) -> np.ndarray:
    """Bytes of the nearest e4m3 values of u >= 0 (at most 448), ties to the even byte; NaN for NaN."""
    grid = E4M3[:127]
    v = np.minimum(u.astype(np.float64), 448.0)
    hi = np.clip(np.searchsorted(grid, v), 1, 126)
    lo = hi - 1
    down, up = v - grid[lo], grid[hi] - v
    out = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    return np.where(np.isnan(u), 127, out).astype(np.uint8)


def power_above(a, top) -> np.ndarray:
    """Exponents k of the smallest 2^k with a <= top * 2^k (a > 0)."""
    m, e = np.frexp(a)
    mt, et = np.frexp(top)
    return (e - et + (m > mt)).astype(np.int64)


def tensor_factor(x) -> float:
    x = np.abs(x[np.isfinite(x)])
    a = x.max() if x.size else 0.0
    return 0.0 if a == 0 else 2.0 ** float(power_above(a, 2688.0))


def quantize(x, fmt, factor=None):
    """(codes, scale bytes) of x (R x C, fp32 values) with blocks along its rows; codes are 255 where a block's scale is NaN.  Every step as the header
    has it, in fp32."""
    f = np.float32
    R, C = x.shape
    nb = BLOCK[fmt]
    wide = np.zeros((R, blocks(C, fmt) * nb), f)
    wide[:, :C] = x
    b = wide.reshape(R, -1, nb)
    with np.errstate(all="ignore"):
        amax = np.where(np.isfinite(b).all(-1), np.abs(b).max(-1), f("nan")).astype(f)
        if fmt == "nvfp4":
            g = f(1) / f(factor) if factor >= 2.0 ** -100 else f(0)
            s = nearest_e4m3((amax * g).astype(f) * (f(1) / f(6)))
            step = (E4M3[s].astype(f) * f(factor)).astype(f)
        else:
            k = np.where(amax > 0, power_above(np.where(amax > 0, amax, 1.0).astype(np.float64), 6.0), -127)
            s = np.where(np.isnan(amax), 255, np.clip(k, -127, 127) + 127).astype(np.uint8)
            step = scale_values(s, fmt)
        some = step > 0
        v = np.where(some[..., None], b / np.where(some, step, 1)[..., None].astype(b.dtype if fmt == "nvfp4" else np.float64), b * 0)
        c = nearest_code(v)
    c = np.where(np.isnan(amax)[..., None], 255, c)
    return c.reshape(R, -1)[:, :C], s


def product_bound(magnitude, depth, out_dtype, exact, extra=0.0) -> np.ndarray:
    """Largest error of a result: every addition of the contraction in 32 bits, each off by 2^-23 of the sum of magnitudes (which covers truncation as
    well as rounding), three products with factors, then one rounding to the result's type."""
    inner = (depth + 4) * 2.0 ** -23 * (magnitude + extra)
    return inner + UNIT[out_dtype] * (np.abs(exact) + inner) + SMALLEST[out_dtype]


def check_product(got, p, q, what="", before=None):
    """got against p @ q.T (+ before), element by element."""
    exact = p @ q.T
    mag = np.abs(p) @ np.abs(q).T
    if before is not None:
        exact, mag = exact + before, mag + np.abs(before)
    bound = product_bound(mag, p.shape[1], got.dtype, exact)
    g = f64(got)
    off = np.abs(g - exact)
    # a result that rounds past the type's largest number is an infinity: past the midpoint to the next power of two's grid
    over = torch.finfo(got.dtype).max * (1 + UNIT[got.dtype] / 2)
    past = np.isinf(g) & (np.sign(g) == np.sign(exact)) & (np.abs(exact) + bound >= over)
    bad = ~((off <= bound) | past)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} off, first at {np.argwhere(bad)[0]}: off {off[bad][0]:.3g}, bound {bound[bad][0]:.3g}"
