"""Definitions of the few-bit operators, in fp64 and whole numbers.

TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).

  quant_i8 / rmsnorm   a token's values as int8 times one scale, with and without the root-mean-square
                       norm in front; the int8 value is the exact nearest integer of 127 x / max|x|
                       (ties to even), which does not depend on the norm's factor
  gemm_i8_scaled       exact integer sums, then three fp32 roundings and one to fp16
  mx4_*                blocks of 32 rows in e2m1 with one power of two
"""
from __future__ import annotations

from fractions import Fraction

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32


def _round_ratio(a: np.ndarray, top: float) -> np.ndarray:
    """Nearest integers of 127 a / top, ties to even (fp64: the quotient of a 29-bit and a 22-bit number
    is never within 2^-24 of a half unless it is one, and a half is exact)."""
    return np.rint(127.0 * a / top)


def round_ratio_exact(a: float, top: float) -> int:
    """The same for one value with rational numbers."""
    return round(Fraction(float(a)) * 127 / Fraction(float(top)))


def quant_i8(X16: np.ndarray):
    """X: M x K fp16 (one token a row) -> int8 values M x K and fp64 scales."""
    return _quant(X16.astype(np.float64), np.ones(X16.shape[0]))


def _quant(g: np.ndarray, inv: np.ndarray):
    M = g.shape[0]
    q, scale = np.zeros(g.shape, np.int8), np.zeros(M)
    for m in range(M):
        if not np.isfinite(g[m]).all():
            scale[m] = np.nan
            continue
        top = np.abs(g[m]).max()
        if top > 0:
            q[m] = _round_ratio(g[m], top).astype(np.int8)
            scale[m] = top * inv[m] / 127.0
    return q, scale


def rmsnorm(X16, R16=None, gamma16=None, eps=1e-6):
    """M x K fp16 -> h (fp16), y (fp64), int8 values, fp64 scales."""
    h = X16 if R16 is None else (X16.astype(np.float64) + R16.astype(np.float64)).astype(np.float16)
    h64 = h.astype(np.float64)
    g = h64 if gamma16 is None else h64 * gamma16.astype(np.float64)
    with np.errstate(all="ignore"):
        inv = 1.0 / np.sqrt((h64 * h64).mean(axis=1) + eps)
        y = g * inv[:, None]
    q, scale = _quant(g, inv)
    return h, y, q, scale


def gemm_i8_scaled(sums: np.ndarray, a_scale: np.ndarray, w_scale: np.ndarray) -> np.ndarray:
    """sums: M x N exact integers; the product of the two fp32 scales, of that and the fp32 sum, and the result to
    fp16, each rounded once."""
    f = a_scale.astype(np.float32)[:, None] * w_scale.astype(np.float32)[None, :]
    with np.errstate(all="ignore"):
        return (sums.astype(np.float32) * f).astype(np.float16)


# ---- microscaled 4-bit ------------------------------------------------------------------------
def mx4_block(x):
    """One block (up to 32 finite values) by search: (scale byte, list of codes)."""
    top = max((abs(float(v)) for v in x), default=0.0)
    if top == 0.0:
        return 127, [8 if np.signbit(v) else 0 for v in x]
    e = -40
    while 2.0 ** (e + 1) <= top:
        e += 1
    e -= 2
    codes = []
    for v in x:
        t = Fraction(abs(float(v))) / Fraction(2) ** e
        d = [abs(t - Fraction(float(g))) for g in E2M1]
        best = min(d)
        near = [c for c in range(8) if d[c] == best]
        c = near[0] if len(near) == 1 else [c for c in near if c % 2 == 0][0]
        codes.append(c | (8 if np.signbit(v) else 0))
    return e + 127, codes


def mx4_quant(X: np.ndarray):
    """K x M fp16 -> codes ceil(K/32) x M x 32 (uint8, 0..15), scale bytes ceil(K/32) x M.  Blocks with an infinity or
    NaN: scale 255, codes 0."""
    K, M = X.shape
    KB = -(-K // BLOCK)
    b = np.zeros((KB * BLOCK, M))
    b[:K] = X.astype(np.float64)
    b = b.reshape(KB, BLOCK, M)
    bad = ~np.isfinite(b).all(axis=1)
    b = np.where(bad[:, None, :], 0.0, b)
    top = np.abs(b).max(axis=1)
    e = np.where(top > 0, np.frexp(top)[1] - 3, 0)
    t = np.abs(b) / np.exp2(e.astype(np.float64))[:, None, :]
    codes = np.zeros(b.shape, np.uint8)
    for c in range(7):
        mid = (E2M1[c] + E2M1[c + 1]) / 2
        codes += ((t > mid) | ((t == mid) & ((c + 1) % 2 == 0))).astype(np.uint8)
    codes |= (np.signbit(b) * 8).astype(np.uint8)
    scale = np.where(bad, 255, e + 127).astype(np.uint8)
    codes[np.broadcast_to(bad[:, None, :], codes.shape)] = 0
    return np.ascontiguousarray(codes.transpose(0, 2, 1)), scale


def mx4_values(codes: np.ndarray, scale: np.ndarray, K: int) -> np.ndarray:
    """K x M fp64 of codes KB x M x 32 and scale bytes KB x M."""
    v = E2M1[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(scale == 255, np.nan, np.exp2(scale.astype(np.float64) - 127))
    v = v * s[:, :, None]
    KB, M, _ = v.shape
    return v.transpose(0, 2, 1).reshape(KB * BLOCK, M)[:K]


def mx4_bytes(codes: np.ndarray) -> np.ndarray:
    """Codes KB x M x 32 -> bytes KB x M x 16, the even row in the low half of a byte."""
    return (codes[:, :, 0::2] | (codes[:, :, 1::2] << 4)).astype(np.uint8)


def mx4_kept_rows(mask: np.ndarray, G: int):
    """Kept columns, and per tile of G of them the 0/1 rows of the blocks that keep anything there."""
    cols = np.flatnonzero(mask.any(axis=0))
    K = mask.shape[0]
    tiles = []
    for i in range(0, cols.size, G):
        rows = mask[:, cols[i:i + G]].any(axis=1)
        keep = np.zeros(K, bool)
        for b in range(0, K, BLOCK):
            keep[b:b + BLOCK] = rows[b:b + BLOCK].any()
        tiles.append(keep)
    return cols, tiles


def mx4_weight(B16: np.ndarray, mask: np.ndarray) -> np.ndarray:
    """What a packed weight stands for (K x N fp64)."""
    Bm = np.where(mask != 0, B16, np.float16(0))
    return mx4_values(*mx4_quant(Bm), B16.shape[0])


def gemm_mx4(codes, scale, B16, mask, G):
    """N x M fp64: over the blocks that a tile keeps (so that a NaN block of a token reaches those columns only)."""
    K, N = B16.shape
    A, W = mx4_values(codes, scale, K), mx4_weight(B16, mask)
    cols, tiles = mx4_kept_rows(mask, G)
    C = np.zeros((N, A.shape[1]))
    with np.errstate(all="ignore"):
        for t, keep in enumerate(tiles):
            tc = cols[t * G:(t + 1) * G]
            C[tc] = W[np.ix_(keep, tc)].T @ A[keep]
    return C
