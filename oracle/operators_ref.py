"""Plain float64 reference of dropout, LayerNorm with its residual add, and matrices in 8-bit floats.

TEST INFRASTRUCTURE ONLY (see the package docstring).  The definitions are those of include/layup.h.
"""
from __future__ import annotations

import numpy as np

U32 = 2.0 ** -24  # half a step of float32, relative
TOPS = {"e4m3": (8, 3, -6), "e5m2": (15, 2, -14)}  # exponent of the largest value, mantissa bits, least exponent


def philox4x32_10(ctr, key):
    """ctr: four arrays of 32-bit words, key: two words; the four output words."""
    c = [np.asarray(x, np.uint64) for x in ctr]
    k = [int(key[0]), int(key[1])]
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), p1 & low,
             (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p0 & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def drop_threshold(p):
    return min(65535, int(np.floor(float(np.float32(p)) * 65536 + 0.5)))


def drop_scale(p):
    return 65536.0 / (65536 - drop_threshold(p))


def keep_mask(rows, cols, p, seed, offset, row0=0):
    """Truth values [rows, cols]; row0: number of the first row."""
    groups = -(-cols // 8)
    g, r = np.meshgrid(np.arange(groups), row0 + np.arange(rows))
    offset &= (1 << 64) - 1
    w = philox4x32_10([g, r, np.full_like(g, offset & 0xFFFFFFFF), np.full_like(g, offset >> 32)],
                      [seed & 0xFFFFFFFF, seed >> 32])
    half = [x >> np.uint64(16) if h else x & np.uint64(0xFFFF) for x in w for h in (0, 1)]
    return np.stack(half, -1).reshape(rows, 8 * groups)[:, :cols] >= drop_threshold(p)


def dropout(x, p, seed, offset):
    x = np.asarray(x, np.float64)
    if drop_threshold(p) == 0:
        return x.copy()
    return np.where(keep_mask(*x.shape, p, seed, offset), x * drop_scale(p), 0.0)


def norm_fwd(s, gamma, beta, eps):
    """(y, mean, rstd) of the rows of s."""
    s = np.asarray(s, np.float64)
    mean = s.mean(1)
    rstd = 1.0 / np.sqrt(((s - mean[:, None]) ** 2).mean(1) + eps)
    return (s - mean[:, None]) * rstd[:, None] * gamma + beta, mean, rstd


def norm_bwd(dy, s, mean, rstd, gamma, dsum):
    """(ds, dgamma, dbeta), from the given statistics."""
    xh = (s - mean[:, None]) * rstd[:, None]
    a = dy * gamma
    ds = dsum + rstd[:, None] * (a - a.mean(1, keepdims=True) - xh * (a * xh).mean(1, keepdims=True))
    return ds, (dy * xh).sum(0), dy.sum(0)


def round_fp8(v, fmt):
    """Finite values within the format, rounded to nearest, ties to even."""
    _, bits, least = TOPS[fmt]
    v = np.asarray(v, np.float64)
    _, e = np.frexp(v)
    step = np.ldexp(1.0, np.maximum(e - 1, least) - bits)
    return np.rint(v / step) * step


def quantise(x, fmt, block_rows):
    """(values as float64, NaN where x is not finite; scale bytes [row blocks, column blocks])."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    nr, nc = -(-rows // block_rows), -(-cols // 128)
    top = TOPS[fmt][0]
    e = np.zeros((nr, nc), np.int64)
    q = np.empty_like(x)
    fin = np.isfinite(x)
    for i in range(nr):
        for j in range(nc):
            at = (slice(i * block_rows, (i + 1) * block_rows), slice(j * 128, (j + 1) * 128))
            a = np.max(np.where(fin[at], np.abs(x[at]), 0.0), initial=0.0)
            if a > 0:
                k = -126
                while a > np.ldexp(1.75 * 2.0 ** top, k):
                    k += 1
                e[i, j] = k
            q[at] = np.where(fin[at], round_fp8(np.where(fin[at], np.ldexp(x[at], -e[i, j]), 0.0), fmt), np.nan)
    return q, (e + 127).astype(np.uint8)


def quantise_all(x, fmt, block_rows):
    """quantise, all blocks at once: amax = m 2^e with 1/2 <= m < 1 has the exponent e - 1 - top, one more above 7/8."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    nr, nc = -(-rows // block_rows), -(-cols // 128)
    fin = np.isfinite(x)
    t = np.zeros((nr * block_rows, nc * 128))
    t[:rows, :cols] = np.abs(np.where(fin, x, 0.0))
    m, e = np.frexp(t.reshape(nr, block_rows, nc, 128).max((1, 3)))
    e = np.where(m > 0, np.maximum(e - 1 - TOPS[fmt][0] + (m > 0.875), -126), 0).astype(np.int64)
    each = np.repeat(np.repeat(e, block_rows, 0)[:rows], 128, 1)[:, :cols]
    return np.where(fin, round_fp8(np.ldexp(np.where(fin, x, 0.0), -each), fmt), np.nan), (e + 127).astype(np.uint8)


def value(q, scale, block_rows):
    """The values that 8-bit values and scale bytes stand for."""
    rows, cols = q.shape
    e = scale.astype(np.int64) - 127
    return np.ldexp(q, np.repeat(np.repeat(e, block_rows, 0)[:rows], 128, 1)[:, :cols])
