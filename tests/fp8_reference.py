"""Plain 64-bit forms of the 8-bit products with block scales and of their quantiser, for the tests (numpy; shares no code with the library)."""
from __future__ import annotations

import numpy as np
import torch

FP8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
FP8_MAX = {"e4m3": 448.0, "e5m2": 57344.0}
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}     # half an ulp, relative
SMALLEST = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}   # half the smallest subnormal


def f64(t) -> np.ndarray:
    return t.detach().float().cpu().numpy().astype(np.float64)


def spread(s, rows, cols, R, C) -> np.ndarray:
    """Scales of rows x cols blocks, one for each element of an R x C matrix."""
    s = np.asarray(s, dtype=np.float64)
    return np.repeat(np.repeat(s, rows, -2)[..., :R, :], cols, -1)[..., :C]


def values(q, s, rows, cols) -> np.ndarray:
    v = f64(q)
    return v * spread(f64(s), rows, cols, *v.shape[-2:])


def codes(fp8: str) -> np.ndarray:
    """Every finite value of the type, ascending."""
    all_codes = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(FP8[fp8])
    v = f64(all_codes)
    return np.unique(v[np.isfinite(v)])


def nearest(v, fp8: str) -> np.ndarray:
    """v rounded to the nearest finite value of the type, ties to the code with an even mantissa."""
    grid = codes(fp8)
    v = np.clip(v, grid[0], grid[-1])
    hi = np.clip(np.searchsorted(grid, v), 1, len(grid) - 1)
    lo = hi - 1
    down, up = v - grid[lo], grid[hi] - v
    half = len(grid) // 2                      # index of zero: a code's parity is that of its distance from it
    even_lo = (lo - half) % 2 == 0
    return np.where((down < up) | ((down == up) & even_lo), grid[lo], grid[hi])


def quantize(x, rows, cols, fp8: str, pow2: bool):
    """(values x / scale before rounding, scales) by the definition; x in 64 bits."""
    R, C = x.shape
    top = FP8_MAX[fp8]
    nr, nc = -(-R // rows), -(-C // cols)
    s = np.ones((nr, nc))
    zero = np.zeros((nr, nc), dtype=bool)
    for i in range(nr):
        for j in range(nc):
            b = np.abs(x[i * rows:(i + 1) * rows, j * cols:(j + 1) * cols])
            b = b[np.isfinite(b)]
            a = b.max() if b.size else 0.0
            if a < 2.0 ** -100:
                zero[i, j] = True
                continue
            s[i, j] = a / top
            if pow2:
                m, e = np.frexp(s[i, j])
                s[i, j] = 2.0 ** (e - 1 if m == 0.5 else e)
    full = spread(s, rows, cols, R, C)
    v = np.where(spread(zero, rows, cols, R, C) > 0, x * 0.0, x / full)
    return np.where(np.isfinite(x), v, np.nan), s


def product_bound(magnitude, blocks: int, out_dtype, exact) -> np.ndarray:
    """Largest error of a result: 128 additions inside a block and four operations per block in 32 bits (each 2^-23 of the sum
    of magnitudes, which covers truncation as well as rounding), then one rounding to the result's type."""
    inner = (128 + 4 * blocks) * 2.0 ** -23 * magnitude
    return inner + UNIT[out_dtype] * (np.abs(exact) + inner) + SMALLEST[out_dtype]


def check_product(got, p, q, blocks, what=""):
    """got against p @ q.T of the scaled operands, element by element."""
    exact = p @ q.T
    bound = product_bound(np.abs(p) @ np.abs(q).T, blocks, got.dtype, exact)
    off = np.abs(f64(got) - exact)
    bad = ~(off <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} off, first at {np.argwhere(bad)[0]}: off {off[bad][0]:.3g}, bound {bound[bad][0]:.3g}"
