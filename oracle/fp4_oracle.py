"""Plain CPU definitions of matrices in 4-bit floating point with a scale for each block of 32, in 64 bits.  Test infrastructure:
shares no code with the CUDA library."""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])     # by code: one mantissa bit, so even codes have mantissa 0


def scale_of(amax):
    """The smallest power of two 2^e with amax <= 6 * 2^e, amax taken as at least 2^-100; NaN where amax is not finite."""
    if not np.isfinite(amax):
        return np.nan
    amax, e = max(float(amax), 2.0 ** -100), -110
    while amax > 6.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def to_e2m1(v):
    """v (|v| <= 6) to the nearest value, ties to the even code."""
    a = np.abs(v)
    hi = np.searchsorted(GRID, a).clip(1, 7)
    lo = hi - 1
    below, above = a - GRID[lo], GRID[hi] - a
    code = np.where(below < above, lo, np.where(above < below, hi, np.where(lo % 2 == 0, lo, hi)))
    return np.copysign(GRID[code], v)


def quantize(x):
    """(codes [rows, cols], scales [rows, blocks])"""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    codes, scales = np.zeros_like(x), np.empty((rows, -(-cols // 32)))
    for r in range(rows):
        for b in range(scales.shape[1]):
            block = x[r, 32 * b:32 * b + 32]
            scales[r, b] = scale_of(np.abs(block).max())
            if np.isfinite(scales[r, b]):
                codes[r, 32 * b:32 * b + 32] = to_e2m1(block / scales[r, b])
    return codes, scales


def dequantize(codes, scales):
    return codes * np.repeat(scales, 32, 1)[:, :codes.shape[1]]
