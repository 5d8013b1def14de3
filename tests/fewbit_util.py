"""Helpers of the few-bit tests: activations with awkward values, masks, device calls, error bounds.

Bounds (relative to exact fp64 values; half a step of fp16 is 2^-11 of the value, 2^-25 below its normal range):
  norm   fp32: a lane adds up to ceil(K/128) squares in a row, then 4 + 8 more in a tree, all positive: at most
         (K/128 + 13) * 2^-24 of the sum, half of that in its square root; the mean, the sum with eps, root, reciprocal and the
         two or three products are one rounding each.  (K/128 + 32) * 2^-24 covers both outputs.
  mx4    products of codes and scales are exact; every addition of n of them may lose a step of fp32, 2^-23 of the
         running sum, which is at most S = |A| . |W|: n * 2^-23 * S, and the rounding to fp16.
"""
import numpy as np

from oracle import fewbit as ofb

STEP16 = 2.0 ** -11


def up(x, a):
    return -(-x // a) * a


def acts(seed, M, K, sigma=1.0):
    """M x K fp16 with rows of different size, zeros, subnormal numbers, ties and a token of zeros."""
    rng = np.random.default_rng(seed)
    x = (rng.standard_normal((M, K)) * sigma * np.exp(rng.standard_normal((1, K)))).astype(np.float16)
    x[:, rng.random(K) < 0.05] = 0
    if M > 2:
        x[M // 2] = 0
        x[M - 1] = (rng.integers(-40, 41, K) * 2.0 ** -24).astype(np.float16)      # subnormal
    if M > 3:
        x[1] = (rng.integers(-8, 9, K) / 8.0).astype(np.float16)                   # halves of a quotient in plenty
    return x


def norm_tol(K):
    return (K / 128 + 32) * 2.0 ** -24


def dev_km(X, ld, pad=np.nan):
    """M x K array -> device K x ld."""
    import torch
    M, K = X.shape
    t = np.full((K, ld), pad, X.dtype)
    t[:, :M] = X.T
    return torch.from_numpy(t).cuda()


def block_mask(rng, K, N, G, col_keep=0.8, block_keep=0.5):
    """Tiles of G kept columns that keep random blocks of 32 rows."""
    cols = np.flatnonzero(rng.random(N) < col_keep)
    mask = np.zeros((K, N), np.uint8)
    for i in range(0, cols.size, G):
        for b in range(0, K, 32):
            if rng.random() < block_keep:
                mask[b:b + 32, cols[i:i + G]] = 1
    return mask


def assert_mx4_close(C, codes, scale, B16, mask, G):
    """C: N x M.  NaN exactly where the definition has it, else the bound above."""
    K = B16.shape[0]
    ref = ofb.gemm_mx4(codes, scale, B16, mask, G)
    A, W = np.abs(ofb.mx4_values(codes, scale, K)), np.abs(ofb.mx4_weight(B16, mask))
    C = C.astype(np.float64)
    nan = np.isnan(ref)
    assert np.array_equal(nan, np.isnan(C))
    S = W.T @ np.nan_to_num(A)
    assert np.abs(ref[~nan]).max(initial=0.0) < 65000
    err = np.abs(np.where(nan, 0.0, C - ref))
    allowed = np.abs(ref) * STEP16 + K * 2.0 ** -23 * S * (1 + STEP16) + np.where(S > 0, 2.0 ** -25, 0.0)
    bad = ~nan & (err > allowed)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist())


def quant_mx4_dev(tw, X, layout, stream=0, ldq=None):
    """X: M x K fp16.  Returns device codes (nb x ldq x 16) and scale bytes (nb x ldq)."""
    import torch
    M, K = X.shape
    nb, ldq = up(K, 32) // 32, ldq or up(M, 16)
    if layout == tw.LAYOUT_KM:
        ldx = up(M, 8)
        Xd = dev_km(X, ldx)
    else:
        ldx = up(K, 8)
        t = np.full((M, ldx), np.nan, np.float16)
        t[:, :K] = X
        Xd = torch.from_numpy(t).cuda()
    Q = torch.full((nb, ldq, 16), 0xA5, dtype=torch.uint8, device="cuda")
    S = torch.full((nb, ldq), 0xA5, dtype=torch.uint8, device="cuda")
    tw.tw_quant_mx4(Xd.data_ptr(), M, K, ldx, layout, Q.data_ptr(), S.data_ptr(), ldq, stream)
    torch.cuda.synchronize()
    return Q, S
