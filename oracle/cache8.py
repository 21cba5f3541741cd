"""The 8-bit KV cache, written out from its definition (oracle side).

TEST INFRASTRUCTURE ONLY; shares no code with the HIP library.

Tiles of 32 tokens; per tile, KV head and K or V: scale = max |x| (1 / M) in 32 bits, rounded up to 12 significant bits, code = x / scale
to nearest, ties to even (whole numbers for M = 127, E4M3 numbers for M = 448).  A last tile that is not full is held as it came.
Exact: scales and codes have few enough bits for fp64, and the rounding decisions are made on Fractions where fp64 would round.
"""
import math

import numpy as np

TILE = 32
MOST = {"int8": 127, "e4m3": 448}


def scale_of(a, fmt):
    """a: the largest magnitude (exact).  fp64 value of the fp32 scale."""
    if not np.isfinite(a):
        return math.nan
    if a == 0:
        return 0.0
    s = float(np.float32(np.float32(a) * np.float32(1.0 / MOST[fmt])))
    m, e = math.frexp(s)                                     # 0.5 <= m < 1
    return math.ldexp(math.ceil(m * 4096), e - 12)


def quantise_tile(x, fmt):
    """x [32][d] (fp16 values) -> (codes as the numbers that they stand for, fp64 [32][d]; scale)."""
    x = np.asarray(x, dtype=np.float64)
    s = scale_of(np.abs(x).max(), fmt)
    if not s > 0:
        return np.zeros_like(x), s
    y = x / s                                                # 11 by 12 bits: fp64 is on the right side of every boundary
    if fmt == "int8":
        return np.rint(y), s
    e = np.maximum(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -40))), -6)
    e = np.where(np.abs(y) >= 2.0 ** (e + 1), e + 1, np.where((np.abs(y) < 2.0 ** e) & (e > -6), e - 1, e))
    step = 2.0 ** (e - 3)
    return np.rint(y / step) * step, s


def held(rows, fmt, n_codes):
    """What the cache holds of rows [n][G][d]: the first n_codes tokens (a multiple of 32) as their codes say, the others as they came."""
    out = np.asarray(rows, dtype=np.float64).copy()
    for t in range(n_codes // TILE):
        for g in range(out.shape[1]):
            codes, s = quantise_tile(out[t * TILE:(t + 1) * TILE, g], fmt)
            out[t * TILE:(t + 1) * TILE, g] = codes * s
    return out


def unpack(codes, scales, *, G, gg, d, T, fmt, page, tile):
    """One tile of one layer from the raw bytes of the buffers, from the layout's description: fp64 [2][32][G][d]."""
    out = np.empty((2, TILE, G, d))
    for g in range(G):
        for kv in range(2):
            at = ((page * (T // TILE) + tile) * G * 2 + (g // gg) * 2 * gg + kv * gg + g % gg) * TILE * d
            s = float(scales.reshape(-1)[((page * (T // TILE) + tile) * G + g) * 2 + kv])
            for key in range(TILE):
                for e in range(d):
                    if kv == 0:
                        h, c, q, i = key // 16, e // 32, e % 32 // 8, e % 8
                        j, p, lane = (2 * h + c // 2, c % 2, 16 * q + key % 16) if d == 128 else (h, c, 16 * q + key % 16)
                    else:
                        half, q, i = key // 16, key % 16 // 4, key % 4
                        i, j, p, lane = i + 4 * half, e // 32, e // 16 % 2, 16 * q + e % 16
                    out[kv, key, g, e] = value(codes.reshape(-1)[at + 16 * (64 * j + lane) + 8 * p + i], fmt) * s
    return out


def value(byte, fmt):
    byte = int(byte)
    if fmt == "int8":
        return byte - 128
    sign, e, m = (-1.0 if byte & 128 else 1.0), byte >> 3 & 15, byte & 7
    if e == 15 and m == 7:
        return math.nan
    return sign * (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))


def attend(q, rows_k, rows_v, n, fmt, appends):
    """q [H][d], rows [>= n][G][d] -> fp64 [H][d] over n keys."""
    H, d = q.shape
    if n == 0:
        return np.zeros((H, d))
    G = rows_k.shape[1]
    codes = (n - (1 if appends else 0)) // TILE * TILE
    k, v = held(rows_k[:n], fmt, codes), held(rows_v[:n], fmt, codes)
    out = np.empty((H, d))
    for h in range(H):
        g = h // (H // G)
        s = k[:, g] @ np.asarray(q[h], dtype=np.float64) / math.sqrt(d)
        w = np.exp(s - s.max())
        out[h] = w @ v[:, g] / w.sum()
    return out
