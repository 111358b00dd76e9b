"""Plain CPU definitions of the operators around the tied weight, in 64 bits (dropout, embedding, 8-bit matrices and
their product, sampling).  Test infrastructure: shares no code with the CUDA library."""
from __future__ import annotations

import numpy as np

LOW = np.uint64(0xFFFFFFFF)


def philox4x32(counter, key):
    """Ten rounds of Philox4x32 on Python integers: the published round function, one word at a time."""
    c0, c1, c2, c3 = counter
    k0, k1 = key
    for _ in range(10):
        p0, p1 = 0xD2511F53 * c0, 0xCD9E8D57 * c2
        c0, c1, c2, c3 = (p1 >> 32) ^ c1 ^ k0, p1 & 0xFFFFFFFF, (p0 >> 32) ^ c3 ^ k1, p0 & 0xFFFFFFFF
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c0, c1, c2, c3


def drop_factor(rows, d, p, seed, offset=0, row_offset=0):
    """[rows, d] of 0 (dropped) or 65536 / (65536 - cut)."""
    cut = int(np.rint(p * 65536))
    if cut >= 65536:
        return np.zeros((rows, d))
    groups = -(-d // 8)
    shape = (rows, groups)
    c = [np.broadcast_to(np.arange(groups, dtype=np.uint64), shape),
         np.broadcast_to(np.arange(row_offset, row_offset + rows, dtype=np.uint64)[:, None], shape),
         np.full(shape, offset & 0xFFFFFFFF, np.uint64), np.full(shape, (offset >> 32) & 0xFFFFFFFF, np.uint64)]
    k0, k1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    s = np.uint64(32)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> s) ^ c[1] ^ np.uint64(k0), b & LOW, (a >> s) ^ c[3] ^ np.uint64(k1), a & LOW]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    halves = np.stack([h for w in c for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], -1).reshape(rows, groups * 8)
    return np.where(halves[:, :d] >= np.uint64(cut), 65536.0 / (65536 - cut), 0.0)


def e4m3_values():
    """The value of every 8-bit code (4 exponent bits, bias 7, 3 mantissa bits; 0x7F and 0xFF are NaN)."""
    v = np.empty(256)
    for code in range(256):
        e, m = (code >> 3) & 15, code & 7
        x = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v[code] = np.nan if code & 127 == 127 else -x if code & 128 else x
    return v


def to_e4m3(x):
    """Codes of x (|x| <= 448), to the nearest value, ties to the even code."""
    grid = e4m3_values()[:127]
    a = np.abs(x)
    hi = np.searchsorted(grid, a).clip(1, 126)
    lo = hi - 1
    below, above = a - grid[lo], grid[hi] - a
    code = np.where(below < above, lo, np.where(above < below, hi, np.where(lo % 2 == 0, lo, hi)))
    return (code + np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def quantize(x, block_rows):
    """(codes [rows, cols], scale [column blocks, row blocks]) with blocks of block_rows x 128."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    kb, rb = -(-cols // 128), -(-rows // block_rows)
    blocks = np.zeros((rb * block_rows, kb * 128))
    blocks[:rows, :cols] = x
    blocks = blocks.reshape(rb, block_rows, kb, 128)
    bad = ~np.isfinite(blocks).all((1, 3))
    amax = np.maximum(np.abs(np.where(bad[:, None, :, None], 0, blocks)).max((1, 3)), 2.0 ** -100)
    e = np.full(amax.shape, -120.0)
    while (short := 448 * 2.0 ** e < amax).any():          # the smallest power of two that is large enough
        e += short
    unit = 2.0 ** e
    with np.errstate(invalid="ignore"):
        codes = to_e4m3(np.where(bad[:, None, :, None], 0, blocks) / unit[:, None, :, None])
    return codes.reshape(rb * block_rows, kb * 128)[:rows, :cols], np.where(bad, np.nan, unit).T


def dequantize(codes, scale, block_rows):
    rows, cols = codes.shape
    s = np.repeat(np.repeat(scale.T, block_rows, 0)[:rows], 128, 1)[:, :cols]
    return e4m3_values()[codes] * s


def sample(x, uniform, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, prob, margin): margin is how far, relative to the sums, the nearest decision was from falling otherwise
    (the weights of another exponential differ in their last bits).  z and the fractions are fp32, as defined."""
    f = np.float32
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, np.float64)).astype(f)
    n, top = len(x), x.max()
    if top == -np.inf:
        return -1, 0.0, 1.0
    if not temperature > 0:
        return int(np.argmax(x)), 1.0, 1.0
    with np.errstate(all="ignore"):
        z = np.where(x == top, f(0), (x - top) * (f(1) / f(temperature))).astype(np.float64)
        e = np.where((x == -np.inf) | np.isnan(z), 0.0, np.exp(z))
    w = np.rint(e * 2.0 ** 31)
    margin = 1.0
    order = np.lexsort((np.arange(n), -(x + f(0))))
    if 0 < top_k < n:
        order = order[:top_k]
    if top_p < 1:
        total = w[order].sum()
        upto = max(1.0, np.floor(np.floor(max(top_p, 0) * 2 ** 24) / 2 ** 24 * total))
        before = np.cumsum(w[order]) - w[order]
        if upto > 1:
            margin = min(margin, np.abs(np.cumsum(w[order]) - upto).min() / total)
        order = order[before < upto]
    limit = min(min_p, 1.0)
    if limit > 0:
        others = e[order][e[order] < 1]
        if len(others):
            margin = min(margin, np.abs(others - limit).min())
        order = order[e[order] >= limit]
    order = np.sort(order)
    cum = np.cumsum(w[order])
    at = np.floor(min(np.floor(max(uniform, 0) * 2 ** 24), 2 ** 24 - 1) / 2 ** 24 * cum[-1])
    pick = int(np.searchsorted(cum, at, side="right"))
    if at > 0:
        margin = min(margin, np.abs(cum - at)[w[order] > 0].min() / cum[-1])
    return int(order[pick]), w[order[pick]] / cum[-1], margin
