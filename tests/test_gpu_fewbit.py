"""Few-bit operators on the GPU against their definitions in 64 bits and whole numbers (-m gpu)."""
import numpy as np
import pytest

import paper_2402_10876_amd as tw
from oracle import fewbit as ofb
from oracle import gemm as og
from tests import fewbit_util as fu
from tests.fewbit_util import acts, block_mask, dev_km, up
from tests.helpers import random_tvw_mask, random_tw_mask
import workloads as wl

pytestmark = pytest.mark.gpu


def _stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


# ---- norm and int8 quantiser ---------------------------------------------------------------------
def _norm(X, R, gamma, eps, *, i8, f16, H=True, alias=None, ld=None, ldq=None):
    import torch
    M, K = X.shape
    ld, ldq = ld or up(M, 8), ldq or up(M, 16)
    Xd = dev_km(X, ld)
    Rd = None if R is None else dev_km(R, ld)
    gd = None if gamma is None else torch.from_numpy(gamma).cuda()
    Hd = None if R is None or not H else {"X": Xd, "R": Rd, None: torch.full((K, ld), 7.0, dtype=torch.float16, device="cuda")}[alias]
    Yd = torch.full((K, ld), 7.0, dtype=torch.float16, device="cuda") if f16 else None
    Qd = torch.full((K, ldq), 99, dtype=torch.int8, device="cuda") if i8 else None
    sd = torch.full((M + 3,), 7.0, device="cuda") if i8 else None
    p = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    tw.tw_rmsnorm(p(Xd), p(Rd), p(gd), eps, M, K, ld, p(Hd), p(Yd), p(Qd), ldq, p(sd), _stream())
    torch.cuda.synchronize()
    n = lambda t: None if t is None else t.cpu().numpy()  # noqa: E731
    return n(Hd), n(Yd), n(Qd), n(sd)


def _check_norm(X, R, gamma, eps, **kw):
    M, K = X.shape
    H, Y, Q, s = _norm(X, R, gamma, eps, **kw)
    h, y, q, scale = ofb.rmsnorm(X, R, gamma, eps)
    tol = fu.norm_tol(K)
    if H is not None:
        assert np.array_equal(H[:, :M].T.view(np.uint16), h.view(np.uint16))
        if kw.get("alias") is None:
            assert (H[:, M:] == 7).all()
        else:
            assert np.isnan(H[:, M:]).all()
    if Y is not None:
        fine = np.isfinite(y)
        got = Y[:, :M].T.astype(np.float64)
        err = np.abs(np.where(fine, got - np.where(fine, y, 0), 0))
        assert (err <= np.where(fine, np.abs(np.where(fine, y, 0)), 0) * (fu.STEP16 + tol) * (1 + fu.STEP16) + 2.0 ** -25).all()
        assert np.array_equal(np.isnan(got), np.isnan(y)) and (Y[:, M:] == 7).all()
    if Q is not None:
        assert np.array_equal(Q[:, :M].T, q)
        assert (Q[:, M:] == 99).all() and (s[M:] == 7).all()
        assert np.array_equal(np.isnan(s[:M]), np.isnan(scale))
        assert (np.abs(np.nan_to_num(s[:M] - scale)) <= np.nan_to_num(scale) * tol).all()


@pytest.mark.parametrize("K", [1, 7, 128, 500, 513, 1003, 2048, 2049, 4096, 8200])
@pytest.mark.parametrize("M", [1, 33, 70])
def test_norm(M, K):
    print(f"norm M={M} K={K}", flush=True)
    X, R = acts(M + K, M, K), acts(M + K + 1, M, K, 3.0)
    gamma = (1 + 0.3 * np.random.default_rng(K).standard_normal(K)).astype(np.float16)
    _check_norm(X, R, gamma, 1e-5, i8=True, f16=True)
    _check_norm(X, None, None, 1e-6, i8=True, f16=False)
    _check_norm(X, R, None, 1e-6, i8=False, f16=True, H=False)


@pytest.mark.parametrize("M", list(range(2, 17)) + list(range(1530, 1537)))
def test_norm_of_any_number_of_tokens(M):
    """The last piece of 8 tokens holds 1 to 8 of them; with many long tokens the slices of the rows do."""
    K = 41 if M < 100 else 2100
    print(f"norm M={M} K={K}", flush=True)
    X, R = acts(M + K, M, K), acts(M + K + 1, M, K, 3.0)
    _check_norm(X, R, None, 1e-5, i8=True, f16=True)
    _check_norm(X, R, None, 1e-5, i8=False, f16=True)


@pytest.mark.parametrize("M,K", [(2049, 64), (2500, 1100), (2200, 2100), (4097, 40), (4100, 1030), (4098, 2050), (8200, 300),
                                 (16321, 2049), (16500, 2049), (16450, 96), (8203, 2060), (16397, 1030), (1030, 4200)])
def test_norm_and_quantiser_of_many_tokens(M, K):
    """Every number of tokens per workgroup, with a ragged last one."""
    import torch
    print(f"many tokens M={M} K={K}", flush=True)
    X, R = acts(M + K, M, K), acts(M + K + 1, M, K, 3.0)
    X[M - 2, K // 2] = np.inf
    _check_norm(X, R, None, 1e-5, i8=True, f16=True)
    _check_norm(X, None, None, 1e-5, i8=True, f16=True)
    q, scale = ofb.quant_i8(X)
    Xd, ldq = dev_km(X, up(M, 8)), up(M, 16)
    Q, s = torch.full((K, ldq), 99, dtype=torch.int8, device="cuda"), torch.zeros((M,), device="cuda")
    tw.tw_quant_i8(Xd.data_ptr(), M, K, up(M, 8), Q.data_ptr(), ldq, s.data_ptr(), _stream())
    assert np.array_equal(Q.cpu().numpy()[:, :M].T, q) and (Q[:, M:] == 99).all()
    s = s.cpu().numpy()
    assert np.array_equal(np.isnan(s), np.isnan(scale)) and (np.abs(np.nan_to_num(s - scale)) <= 2.0 ** -23 * np.nan_to_num(scale)).all()


@pytest.mark.parametrize("M,K", [(1, 8193), (19, 8195), (3, 131071), (130, 10000)])
def test_norm_of_few_very_long_tokens(M, K):
    print(f"few long tokens M={M} K={K}", flush=True)
    X, R = acts(M + K, M, K), acts(M + K + 1, M, K, 3.0)
    _check_norm(X, R, None, 1e-5, i8=True, f16=True)
    _check_norm(X, None, None, 1e-5, i8=False, f16=True)
    X[M - 1, K - 1] = np.nan
    _check_norm(X, None, None, 1e-5, i8=True, f16=False)


@pytest.mark.parametrize("M,K", [(1537, 2049), (1001, 3333), (768, 4096), (400, 8200), (79, 2050), (2051, 2500)])
def test_norm_of_long_tokens_in_slices(M, K):
    """With a residual and many rows the work is cut along the rows: every combination of outputs, in place, infinities."""
    print(f"slices M={M} K={K}", flush=True)
    X, R = acts(M + K, M, K), acts(M + K + 1, M, K, 3.0)
    gamma = (1 + 0.3 * np.random.default_rng(K).standard_normal(K)).astype(np.float16)
    _check_norm(X, R, gamma, 1e-5, i8=True, f16=True)
    _check_norm(X, R, gamma, 1e-5, i8=False, f16=True, alias="X", ld=up(M, 8) + 16)
    _check_norm(X, R, None, 1e-5, i8=True, f16=False, alias="R", ldq=up(M, 16) + 32)
    _check_norm(X, R, gamma, 1e-5, i8=True, f16=False, H=False)
    _check_norm(X, R, None, 1e-5, i8=False, f16=True, H=False)
    X[3, 7], X[20, K - 1], R[33, 0], X[M - 1, 130] = np.inf, np.nan, -np.inf, np.nan
    X[40, 5] = R[40, 5] = 60000.0
    _check_norm(X, R, gamma, 1e-5, i8=True, f16=True)
    gamma[K - 2] = np.nan                                 # every token
    _, _, Q, s = _norm(X, R, gamma, 1e-5, i8=True, f16=False)
    assert np.isnan(s[:M]).all() and not Q[:, :M].any()


@pytest.mark.parametrize("K", [5, 1500, 5000])
def test_norm_with_a_gamma_that_is_not_finite(K):
    M = 40
    X = acts(7, M, K)
    for bad in (np.nan, np.inf):
        gamma = np.ones(K, np.float16)
        gamma[K // 2] = bad
        _, _, Q, s = _norm(X, None, gamma, 1e-5, i8=True, f16=False)
        assert np.isnan(s[:M]).all() and not Q[:, :M].any()


@pytest.mark.parametrize("alias", ["X", "R"])
@pytest.mark.parametrize("K", [300, 5000])
def test_norm_in_place_and_wider_strides(alias, K):
    M = 45
    X, R = acts(1, M, K), acts(2, M, K)
    print(f"norm in place {alias} K={K}", flush=True)
    _check_norm(X, R, None, 1e-5, i8=True, f16=True, alias=alias, ld=64, ldq=80)


@pytest.mark.parametrize("K", [200, 3000])
def test_norm_infinities_stay_in_their_token(K):
    M = 50
    X, R = acts(5, M, K), acts(6, M, K)
    gamma = np.ones(K, np.float16)
    X[3, 7], X[20, K - 1], R[33, 0] = np.inf, np.nan, -np.inf
    X[40, 5] = R[40, 5] = 60000.0                         # the sum overflows
    print(f"norm non-finite K={K}", flush=True)
    _check_norm(X, R, gamma, 1e-5, i8=True, f16=True)
    _, _, Q, s = _norm(X, R, gamma, 1e-5, i8=True, f16=False)
    assert np.isnan(s[[3, 20, 33, 40]]).all() and not Q[:, [3, 20, 33, 40]].any() and np.isfinite(s[:M]).sum() == M - 4


def test_norm_largest_and_smallest_values():
    K = 4099
    X = np.zeros((4, K), np.float16)
    X[0], X[1], X[2, 11] = 65504.0, 2.0 ** -24, -65504.0
    X[3] = 1.0
    gamma = np.full(K, 65504.0, np.float16)
    _check_norm(X, None, gamma, 1e-30, i8=True, f16=False)
    _check_norm(X, None, None, 1e-30, i8=True, f16=True)


@pytest.mark.parametrize("M,K", [(1, 1), (5, 31), (40, 768), (33, 1003), (64, 4100), (101, 4200), (1, 8193), (5, 20000)])
def test_quant_i8(M, K):
    import torch
    X = acts(M * 3 + K, M, K)
    if M > 4:
        X[3, K // 2] = np.nan
    ldx, ldq = up(M, 8) + 8, up(M, 16) + 16
    Xd = dev_km(X, ldx)
    Q = torch.full((K, ldq), 99, dtype=torch.int8, device="cuda")
    s = torch.full((M + 1,), 7.0, device="cuda")
    print(f"quant_i8 M={M} K={K}", flush=True)
    tw.tw_quant_i8(Xd.data_ptr(), M, K, ldx, Q.data_ptr(), ldq, s.data_ptr(), _stream())
    q, scale = ofb.quant_i8(X)
    Q, s = Q.cpu().numpy(), s.cpu().numpy()
    assert np.array_equal(Q[:, :M].T, q) and (Q[:, M:] == 99).all() and s[M] == 7
    assert np.array_equal(np.isnan(s[:M]), np.isnan(scale))
    assert (np.abs(np.nan_to_num(s[:M] - scale)) <= 2.0 ** -23 * np.nan_to_num(scale)).all()


def test_the_most_tokens():
    """2^27 tokens of one or two values: the largest grids."""
    import torch
    M = 1 << 27
    x = torch.randn((2, M), device="cuda", dtype=torch.float16)
    Q = torch.zeros((2, M), dtype=torch.int8, device="cuda")
    s = torch.zeros((M,), device="cuda")
    print("most tokens: int8", flush=True)
    tw.tw_quant_i8(x.data_ptr(), M, 2, M, Q.data_ptr(), M, s.data_ptr(), _stream())
    top = x.float().abs().amax(0)
    assert bool((Q.abs().amax(0) == 127 * (top > 0)).all()) and bool(((s * 127 - top).abs() <= 2.0 ** -22 * top).all())
    assert bool((Q.float() * s - x.float()).abs().le(0.5001 * s).all())
    del Q, top
    print("most tokens: norm", flush=True)
    Y = torch.zeros((2, M), dtype=torch.float16, device="cuda")
    tw.tw_rmsnorm(x.data_ptr(), None, None, 1e-6, M, 2, M, None, Y.data_ptr(), None, 0, None, _stream())
    want = x.float() / torch.sqrt((x.float() ** 2).mean(0) + 1e-6)
    assert bool(((Y.float() - want).abs() <= (fu.STEP16 + 1e-5) * want.abs() + 2.0 ** -25).all())
    del Y, want
    print("most tokens: 4 bits", flush=True)
    codes = torch.zeros((1, M, 16), dtype=torch.uint8, device="cuda")
    scale = torch.zeros((1, M), dtype=torch.uint8, device="cuda")
    tw.tw_quant_mx4(x.data_ptr(), M, 2, M, tw.LAYOUT_KM, codes.data_ptr(), scale.data_ptr(), M, _stream())
    at = torch.tensor([0, 1, M // 2 + 3, M - 2, M - 1], device="cuda")
    c, e = ofb.mx4_quant(x[:, at].cpu().numpy())
    assert np.array_equal(codes[0, at].cpu().numpy(), ofb.mx4_bytes(c)[0]) and np.array_equal(scale[0, at].cpu().numpy(), e[0])
    p = tw.tw_pack_mx4(np.array([[1.0], [-2.0]], np.float16), np.ones((2, 1), np.uint8), 64)
    C = torch.zeros((1, M), dtype=torch.float16, device="cuda")
    tw.tw_gemm_mx4(codes.data_ptr(), scale.data_ptr(), M, M, p, C.data_ptr(), M, _stream())
    v = ofb.mx4_values(c, e, 2)
    assert np.array_equal(C[0, at].cpu().numpy(), (v[0] - 2 * v[1]).astype(np.float16))


def test_quant_i8_every_ratio():
    """All pairs of small mantissas: quotients on and next to halves."""
    import torch
    a = np.arange(-1023, 1024).astype(np.float16)
    tops = np.array([1023, 1000, 762, 508, 254, 1022, 511, 2047], np.float16)
    X = np.concatenate([np.clip(a, -t, t)[None] for t in tops]).astype(np.float16)
    X = np.concatenate([X, tops[:, None]], 1)
    M, K = X.shape
    Xd = dev_km(X, 8)
    Q = torch.zeros((K, 16), dtype=torch.int8, device="cuda")
    s = torch.zeros((M,), device="cuda")
    tw.tw_quant_i8(Xd.data_ptr(), M, K, 8, Q.data_ptr(), 16, s.data_ptr(), _stream())
    got = Q.cpu().numpy()[:, :M].T
    for m in range(M):
        assert got[m].tolist() == [ofb.round_ratio_exact(v, tops[m]) for v in X[m]]


# ---- scaled int8 product ---------------------------------------------------------------------------
@pytest.mark.parametrize("pattern", ["tw", "tvw"])
@pytest.mark.parametrize("M,K,N,G", [(1, 100, 70, 64), (37, 300, 333, 128), (300, 210, 300, 64), (700, 1003, 1491, 128),
                                     (2100, 770, 1300, 128), (1500, 2100, 400, 64), (4096, 1024, 2100, 128), (520, 4096, 1024, 128)])
def test_gemm_i8_scaled(M, K, N, G, pattern):
    import torch
    rng = np.random.default_rng(M + K)
    tmask = None
    if pattern == "tw":
        mask = random_tw_mask(rng, K, N, G)
    else:
        mask, tmask = random_tvw_mask(rng, K, N, G)
    A, B = wl.rng_i8(M, (M, K)), wl.rng_i8(K, (K, N))
    lda, ldc = up(M, 16), up(M, 8) + 8
    At = np.full((K, lda), 0x55, np.int8)
    At[:, :M] = A.T
    Ad = torch.from_numpy(At).cuda()
    sa = (rng.random(M) * 0.01).astype(np.float32)
    sw = (rng.random(N) * 0.01).astype(np.float32)
    if M > 3:
        sa[1], sa[2] = 0.0, np.nan                            # a token of zeros, a token that was not finite
    sad, swd = torch.from_numpy(sa).cuda(), torch.from_numpy(sw).cuda()
    C = torch.full((N, ldc), 7.0, dtype=torch.float16, device="cuda")
    p = tw.tw_pack_i8(B, mask, G, tw.PATTERN_TVW if pattern == "tvw" else tw.PATTERN_TW, tile_mask=tmask)
    print(f"gemm_i8_scaled {pattern} M={M} K={K} N={N} G={G}", flush=True)
    tw.tw_gemm_i8_scaled(Ad.data_ptr(), M, lda, p, sad.data_ptr(), swd.data_ptr(), C.data_ptr(), ldc, _stream())
    got = C.cpu().numpy()
    p.free()
    sums = np.rint(A.astype(np.float64) @ (B * (mask != 0)).astype(np.float64))      # whole numbers below 2^53
    want = ofb.gemm_i8_scaled(sums, sa, sw)
    want[:, ~mask.any(0)] = 0                                 # pruned columns: zeros whatever the scales
    assert np.array_equal(got[:, :M].T, want, equal_nan=True)
    assert (got[:, M:] == 7).all()
    assert not np.signbit(got[~mask.any(0), :M]).any()


@pytest.mark.parametrize("M,N", [(50, 300), (900, 1500), (2000, 1500), (4100, 2500), (4090, 3900)])
@pytest.mark.parametrize("tile_m", [0, 64, 128, 256])
def test_int8_tiles_of_every_height(tile_m, M, N):
    """The same whole sums with every height of the tiles, chosen or asked for, in the three types of output."""
    import torch
    rng = np.random.default_rng(M)
    K, G = 200, 128
    mask = random_tw_mask(rng, K, N, G)
    A, B = wl.rng_i8(M, (M, K)), wl.rng_i8(K, (K, N))
    ld = up(M, 16)
    Ad = torch.zeros((K, ld), dtype=torch.int8, device="cuda")
    Ad[:, :M] = torch.from_numpy(np.ascontiguousarray(A.T)).cuda()
    sa, sw = (rng.random(M) * 0.01).astype(np.float32), (rng.random(N) * 0.01).astype(np.float32)
    sad, swd = torch.from_numpy(sa).cuda(), torch.from_numpy(sw).cuda()
    out = [torch.empty((N, ld), dtype=t, device="cuda") for t in (torch.int32, torch.int8, torch.float16)]
    p = tw.tw_pack_i8(B, mask, G, tw.PATTERN_TW)
    print(f"int8 tiles tile_m={tile_m} M={M} N={N}", flush=True)
    tw.tw_set_option("tile_m", tile_m)
    try:
        for dtype in (0, 1):
            tw.tw_gemm_i8(Ad.data_ptr(), M, ld, p, out[dtype].data_ptr(), ld, dtype, 1e-3, _stream())
        tw.tw_gemm_i8_scaled(Ad.data_ptr(), M, ld, p, sad.data_ptr(), swd.data_ptr(), out[2].data_ptr(), ld, _stream())
    finally:
        tw.tw_set_option("tile_m", 0)
    got = [o.cpu().numpy()[:, :M].T for o in out]
    p.free()
    sums = np.rint(A.astype(np.float64) @ (B * (mask != 0)).astype(np.float64))
    assert np.array_equal(got[0], sums.astype(np.int32))
    assert np.array_equal(got[1], np.clip(np.rint(sums.astype(np.float32) * np.float32(1e-3)), -128, 127).astype(np.int8))
    assert np.array_equal(got[2], ofb.gemm_i8_scaled(sums, sa, sw))


@pytest.mark.parametrize("pattern", ["tw", "tvw"])
@pytest.mark.parametrize("M", list(range(193, 201)))
def test_gemm_i8_scaled_of_any_number_of_tokens(M, pattern):
    tw.tw_set_option("tile_m", 64)           # (not the kernel for few tokens)
    try:
        test_gemm_i8_scaled(M, 140, 150, 128, pattern)
    finally:
        tw.tw_set_option("tile_m", 0)


# ---- microscaled 4-bit -----------------------------------------------------------------------------
def _same_codes(Q, S, X, ldq):
    M, K = X.shape
    codes, scale = ofb.mx4_quant(np.ascontiguousarray(X.T))
    Q, S = Q.cpu().numpy(), S.cpu().numpy()
    assert np.array_equal(S[:, :M], scale)
    assert np.array_equal(Q[:, :M], ofb.mx4_bytes(codes))
    assert (Q[:, M:] == 0xA5).all() and (S[:, M:] == 0xA5).all()
    return codes, scale


@pytest.mark.parametrize("layout", ["KM", "MK"])
@pytest.mark.parametrize("M,K", [(1, 1), (1, 32), (2, 31), (33, 33), (130, 300), (64, 1003), (257, 64), (19, 2100), (5003, 700),
                                 (8203, 1030)] + [(M, 77) for M in range(3, 18)])
def test_quant_mx4(M, K, layout):
    X = acts(M + K, M, K)
    if M > 4:
        X[0, K // 2], X[3, 0], X[3, K - 1] = np.inf, np.nan, -np.inf
    print(f"quant_mx4 {layout} M={M} K={K}", flush=True)
    Q, S = fu.quant_mx4_dev(tw, X, getattr(tw, "LAYOUT_" + layout), _stream(), ldq=up(M, 16) + 16)
    _same_codes(Q, S, X, None)


def test_quant_mx4_every_value():
    """Every finite fp16 value as the largest of its block and below maxima of every size."""
    v = np.arange(0x7c00, dtype=np.uint16)
    rng = np.random.default_rng(4)
    cols = [v]
    for shift in (1, 300, 1024, 1500, 2048, 2055, 4096):
        cols.append(np.maximum(v.astype(np.int64) - shift, 0).astype(np.uint16))
    while len(cols) < 32:
        cols.append((v - np.minimum(v, rng.integers(0, 5000, v.size))).astype(np.uint16))
    X = np.stack(cols, 1) | (rng.integers(0, 2, (v.size, 32)) << 15).astype(np.uint16)
    X = X.view(np.float16)
    for layout in (tw.LAYOUT_KM, tw.LAYOUT_MK):
        Q, S = fu.quant_mx4_dev(tw, X, layout, _stream())
        _same_codes(Q, S, X, None)
    X = np.ascontiguousarray(np.concatenate([X, X[:, ::-1], -X], 1))          # (more values than the kernel for few takes)
    Q, S = fu.quant_mx4_dev(tw, X, tw.LAYOUT_KM, _stream())
    _same_codes(Q, S, X, None)


def _gemm_mx4(p, Q, S, M, N, ldc=None):
    import torch
    ldc = ldc or up(M, 8) + 8
    C = torch.full((N, ldc), 7.0, dtype=torch.float16, device="cuda")
    tw.tw_gemm_mx4(Q.data_ptr(), S.data_ptr(), M, Q.shape[1], p, C.data_ptr(), ldc, _stream())
    torch.cuda.synchronize()
    got = C.cpu().numpy()
    assert (got[:, M:] == 7).all()
    return got[:, :M]


MASKS = {
    "blocks": lambda rng, K, N, G: block_mask(rng, K, N, G),
    "all": lambda rng, K, N, G: np.ones((K, N), np.uint8),
    "none": lambda rng, K, N, G: np.zeros((K, N), np.uint8),
    "rows": lambda rng, K, N, G: random_tw_mask(rng, K, N, G, 0.7, 0.1),
    "elements": lambda rng, K, N, G: (rng.random((K, N)) < 0.01).astype(np.uint8),
}


@pytest.mark.parametrize("mask", sorted(MASKS))
@pytest.mark.parametrize("M,K,N,G", [(1, 32, 64, 64), (1, 1000, 333, 128), (31, 33, 40, 128), (64, 4096, 130, 64), (65, 95, 128, 128),
                                     (300, 640, 300, 64), (513, 1003, 515, 128), (130, 31, 1, 128), (1100, 256, 1290, 128)])
def test_gemm_mx4(M, K, N, G, mask):
    rng = np.random.default_rng(M + K + N)
    m = MASKS[mask](rng, K, N, G)
    B = (rng.standard_normal((K, N)) * 0.05 * 2.0 ** rng.integers(-3, 4, (1, N))).astype(np.float16)
    X = acts(M + 1, M, K)
    if M > 4:
        X[2, K // 3] = np.nan                                 # one block of one token
    Q, S = fu.quant_mx4_dev(tw, X, tw.LAYOUT_KM, _stream())
    p = tw.tw_pack_mx4(B, m, G)
    print(f"gemm_mx4 {mask} M={M} K={K} N={N} G={G}", flush=True)
    C = _gemm_mx4(p, Q, S, M, N)
    p.free()
    codes, scale = ofb.mx4_quant(np.ascontiguousarray(X.T))
    fu.assert_mx4_close(C, codes, scale, B, m, G)
    dropped = C[~m.any(0)]
    assert not dropped.any() and not np.signbit(dropped).any()


@pytest.mark.parametrize("G", [64, 128])
@pytest.mark.parametrize("M,K,N", [(20, 3000, 300), (5, 1500, 300), (33, 700, 200), (8199, 1030, 2100), (8199, 500, 1500), (8199, 300, 3200), (3001, 700, 1290), (600, 2000, 900),
                                   (5000, 1030, 2000), (5000, 300, 1300), (1700, 1030, 2000)])
def test_gemm_mx4_of_every_shape(M, K, N, G):
    """Lists of every length for few tokens and the tile shapes of larger products: 512 and 256 rows, 128 rows, tiles of single waves, lists shared among waves."""
    rng = np.random.default_rng(M + K)
    m = block_mask(rng, K, N, G, 1.0, 0.95)
    B = (rng.standard_normal((K, N)) * 0.05).astype(np.float16)
    X = acts(M, M, K)
    X[M - 2, K // 3] = np.inf
    Q, S = fu.quant_mx4_dev(tw, X, tw.LAYOUT_MK, _stream())
    p = tw.tw_pack_mx4(B, m, G)
    print(f"gemm_mx4 M={M} K={K} N={N} G={G}", flush=True)
    C = _gemm_mx4(p, Q, S, M, N)
    p.free()
    codes, scale = ofb.mx4_quant(np.ascontiguousarray(X.T))
    fu.assert_mx4_close(C, codes, scale, B, m, G)


def test_gemm_mx4_of_any_number_of_tokens():
    rng = np.random.default_rng(12)
    K, N, G = 70, 90, 64
    m = block_mask(rng, K, N, G)
    B = (rng.standard_normal((K, N)) * 0.05).astype(np.float16)
    p = tw.tw_pack_mx4(B, m, G)
    for M in range(1, 18):
        X = acts(M, M, K)
        Q, S = fu.quant_mx4_dev(tw, X, tw.LAYOUT_KM, _stream())
        codes, scale = ofb.mx4_quant(np.ascontiguousarray(X.T))
        fu.assert_mx4_close(_gemm_mx4(p, Q, S, M, N), codes, scale, B, m, G)
    p.free()


def test_gemm_mx4_identity_returns_the_weight():
    """One-hot tokens: C is the packed weight exactly, so every lane, block and scale is in its place."""
    rng = np.random.default_rng(8)
    K, N = 320, 260
    B = (rng.standard_normal((K, N)) * 2.0 ** rng.integers(-8, 8, (K, N))).astype(np.float16)
    X = np.eye(K, dtype=np.float16)
    for G in (64, 128):
        mask = block_mask(rng, K, N, G)
        Q, S = fu.quant_mx4_dev(tw, X, tw.LAYOUT_MK, _stream())
        p = tw.tw_pack_mx4(B, mask, G)
        assert np.array_equal(_gemm_mx4(p, Q, S, K, N).T, ofb.mx4_weight(B, mask).astype(np.float16))
        W = p.unpack()[0].view(np.float16)
        assert np.array_equal(W, ofb.mx4_weight(B, mask).astype(np.float16))
        for M in (1, 40):                                     # the kernel for few tokens
            got = _gemm_mx4(p, Q[:, 100:100 + 48].contiguous(), S[:, 100:100 + 48].contiguous(), M, N)
            assert np.array_equal(got.T, W[100:100 + M])
        p.free()


# ---- experts ---------------------------------------------------------------------------------------
def _experts(rng, E, K, N, G, keep=0.6):
    parts, Bs, ms = [], [], []
    for e in range(E):
        m = block_mask(rng, K, N, G, 0.8, keep)
        if e == 1:
            m[:] = 0                                          # an expert of which nothing is left
        B = (rng.standard_normal((K, N)) * 0.05).astype(np.float16)
        parts.append(tw.tw_pack_mx4(B, m, G))
        Bs.append(B)
        ms.append(m)
    return parts, Bs, ms


def _grouped(h, Q, S, M, N, off, ldc=None):
    import torch
    ldc = ldc or up(M, 8) + 8
    C = torch.full((N, ldc), 7.0, dtype=torch.float16, device="cuda")
    o = torch.tensor(off, dtype=torch.int32, device="cuda")
    tw.tw_gemm_mx4_grouped(Q.data_ptr(), S.data_ptr(), M, Q.shape[1], o.data_ptr(), h, C.data_ptr(), ldc, _stream())
    torch.cuda.synchronize()
    return C.cpu().numpy()


@pytest.mark.parametrize("K,N,G,off", [
    (96, 130, 64, [0, 3, 3, 4, 20]),
    (300, 200, 128, [5, 5, 12, 140, 141, 333, 333]),
    (1003, 515, 128, [0, 0, 0, 700]),
    (64, 64, 64, [2, 9]),
    (160, 300, 64, [0, 1000, 1001, 1013, 2100]),
    (96, 130, 128, np.cumsum([0] + list(range(1, 18)) + list(range(70, 78))).tolist()),
    (96, 130, 64, [3] + [12 + 8 * i for i in range(9)] + [141]),
    (200, 600, 128, [0, 1500, 1511, 4000, 4063, 5000, 6200, 7000, 7995]),
    (100, 1500, 64, [0, 1500, 1511, 4000, 4063, 5000, 6200, 7000, 7995]),
    (100, 1500, 128, [0, 1500, 1511, 4000, 4063, 5000, 6200, 7000, 7995]),
    (1030, 2100, 128, [5, 4000, 8190]),
    (500, 1500, 64, [5, 4100, 8390]),
    (1030, 2100, 128, [7, 8300]),
    (128, 128, 128, [0] + sorted(np.random.default_rng(1).integers(0, 400, 79).tolist()) + [400]),
])
def test_grouped(K, N, G, off):
    rng = np.random.default_rng(K + N)
    E, M = len(off) - 1, off[-1] + 5
    parts, Bs, ms = _experts(rng, E, K, N, G)
    h = tw.tw_concat(parts) if E > 1 else parts[0]
    X = acts(K, M, K)
    Q, S = fu.quant_mx4_dev(tw, X, tw.LAYOUT_MK, _stream())
    print(f"grouped E={E} K={K} N={N} G={G} M={M}", flush=True)
    got = _grouped(h, Q, S, M, N, off)
    codes, scale = ofb.mx4_quant(np.ascontiguousarray(X.T))
    assert (got[:, :off[0]] == 7).all() and (got[:, off[-1]:] == 7).all()
    for e in range(E):
        a, b = off[e], off[e + 1]
        if b > a:
            print(f"  expert {e}: {a}..{b}", flush=True)
            fu.assert_mx4_close(got[:, a:b], codes[:, a:b], scale[:, a:b], Bs[e], ms[e], G)
    # the joined weight, side by side
    if E > 1:
        C = _gemm_mx4(h, Q, S, M, N * E)
        fu.assert_mx4_close(C[:N], codes, scale, Bs[0], ms[0], G)
        fu.assert_mx4_close(C[-N:], codes, scale, Bs[-1], ms[-1], G)


@pytest.mark.parametrize("off", [[-5, 4, 4, 30], [0, 20, 10, 99], [50, 40, 30, 20], [7, 7, 7, 7]])
def test_grouped_offsets_outside_are_cut(off):
    """Safe whatever the offsets: nothing behind column M; well-formed ranges are right."""
    rng = np.random.default_rng(3)
    K, N, G, M = 64, 100, 64, 33
    parts, Bs, ms = _experts(rng, 3, K, N, G)
    h = tw.tw_concat(parts)
    X = acts(9, M, K)
    Q, S = fu.quant_mx4_dev(tw, X, tw.LAYOUT_KM, _stream())
    print(f"grouped offsets {off}", flush=True)
    got = _grouped(h, Q, S, M, N, off)
    assert (got[:, M:] == 7).all()
    codes, scale = ofb.mx4_quant(np.ascontiguousarray(X.T))
    cut = [min(max(o, 0), M) for o in off]
    touched = np.zeros(M, int)
    for a, b in zip(cut, cut[1:]):
        touched[a:max(a, b)] += 1
    assert (got[:, :M][:, touched == 0] == 7).all()
    for e, (a, b) in enumerate(zip(cut, cut[1:])):
        if b > a and (touched[a:b] == 1).all():
            fu.assert_mx4_close(got[:, a:b], codes[:, a:b], scale[:, a:b], Bs[e], ms[e], G)


# ---- together --------------------------------------------------------------------------------------
def test_a_layer_in_few_bits_captured_and_replayed():
    """norm -> int8 product -> 4-bit product -> experts -> norm, eager on a stream of its own, then captured and replayed
    with the program's own work in between; every result bit for bit, and the chain against the definitions."""
    import torch
    rng = np.random.default_rng(21)
    M, K, N, G = 150, 200, 264, 64
    ld = up(M, 16)
    X, R = acts(1, M, K), acts(2, M, K)
    gamma = np.ones(K, np.float16)
    B8, m8 = wl.rng_i8(3, (K, N)), random_tw_mask(rng, K, N, G)
    w8 = tw.tw_pack_i8(B8, m8, G)
    B4, m4 = (rng.standard_normal((N, K)) * 0.05).astype(np.float16), block_mask(rng, N, K, G)
    w4 = tw.tw_pack_mx4(B4, m4, G)
    parts, Be, me = _experts(rng, 4, N, K, G)
    we = tw.tw_concat(parts)
    off = [0, 40, 40, 41, M]
    sw = (rng.random(N) * 1e-3 + 1e-4).astype(np.float32)
    dev = "cuda"
    z = lambda *s, dt=torch.float16: torch.zeros(s, dtype=dt, device=dev)  # noqa: E731
    Xd, Rd, gd, swd = dev_km(X, ld, 0), dev_km(R, ld, 0), torch.from_numpy(gamma).cuda(), torch.from_numpy(sw).cuda()
    offd = torch.tensor(off, dtype=torch.int32, device=dev)
    H, Q8, s8, U = z(K, ld), z(K, ld, dt=torch.int8), z(M, dt=torch.float32), z(N, ld)
    nb = up(N, 32) // 32
    Q4, S4, D, E, H2, Y2 = z(nb, ld, 16, dt=torch.uint8), z(nb, ld, dt=torch.uint8), z(K, ld), z(K, ld), z(K, ld), z(K, ld)
    outs = [H, Q8, s8, U, Q4, S4, D, E, H2, Y2]

    def step(st):
        tw.tw_rmsnorm(Xd.data_ptr(), Rd.data_ptr(), gd.data_ptr(), 1e-6, M, K, ld, H.data_ptr(), None, Q8.data_ptr(), ld, s8.data_ptr(), st)
        tw.tw_gemm_i8_scaled(Q8.data_ptr(), M, ld, w8, s8.data_ptr(), swd.data_ptr(), U.data_ptr(), ld, st)
        tw.tw_quant_mx4(U.data_ptr(), M, N, ld, tw.LAYOUT_KM, Q4.data_ptr(), S4.data_ptr(), ld, st)
        tw.tw_gemm_mx4(Q4.data_ptr(), S4.data_ptr(), M, ld, w4, D.data_ptr(), ld, st)
        tw.tw_gemm_mx4_grouped(Q4.data_ptr(), S4.data_ptr(), M, ld, offd.data_ptr(), we, E.data_ptr(), ld, st)
        tw.tw_rmsnorm(D.data_ptr(), E.data_ptr(), None, 1e-6, M, K, ld, H2.data_ptr(), Y2.data_ptr(), None, 0, None, st)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side.cuda_stream)
    torch.cuda.synchronize()
    eager = [o.clone() for o in outs]
    assert all(bool(e.any()) for e in eager)
    # against the definitions, each operator from what the one before it gave
    a = lambda t: t.cpu().numpy()  # noqa: E731
    _, _, q, sc = ofb.rmsnorm(X, R, gamma, 1e-6)
    assert np.array_equal(a(Q8)[:, :M].T, q)
    sums = np.rint(q.astype(np.float64) @ (B8 * (m8 != 0)).astype(np.float64))
    want = ofb.gemm_i8_scaled(sums, a(s8), sw)
    want[:, ~m8.any(0)] = 0
    assert np.array_equal(a(U)[:, :M].T, want)
    codes, scale = ofb.mx4_quant(a(U)[:, :M])
    assert np.array_equal(a(Q4)[:, :M], ofb.mx4_bytes(codes)) and np.array_equal(a(S4)[:, :M], scale)
    fu.assert_mx4_close(a(D)[:, :M], codes, scale, B4, m4, G)
    for e in range(4):
        x, y = off[e], off[e + 1]
        if y > x:
            fu.assert_mx4_close(a(E)[:, x:y], codes[:, x:y], scale[:, x:y], Be[e], me[e], G)
    h2, y2, _, _ = ofb.rmsnorm(a(D)[:, :M].T.copy(), a(E)[:, :M].T.copy(), None, 1e-6)
    assert np.array_equal(a(H2)[:, :M].T, h2)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step(side.cuda_stream)
    torch.cuda.synchronize()
    for replay in range(4):
        for o in outs:
            o.zero_()
        torch.randn((256, 256), device=dev) @ torch.randn((256, 256), device=dev)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for o, e in zip(outs, eager):
            assert torch.equal(o.view(torch.uint8) if o.dtype != torch.float32 else o, e.view(torch.uint8) if e.dtype != torch.float32 else e), replay


def test_long_rows_pass_32_bit_offsets():
    """Rows of activations and of C more than 2^32 bytes from the first."""
    import torch
    if torch.cuda.get_device_properties(0).total_memory < 60 << 30:
        pytest.skip("needs 30 GiB of device memory")
    M, K, N, G = 40, 160, 96, 64
    ld = 1 << 25                                           # 5 block rows of 512 MiB of codes, C rows of 64 MiB
    rng = np.random.default_rng(2)
    X = acts(3, M, K)
    Xd = torch.zeros((K, ld), dtype=torch.float16, device="cuda")
    Xd[:, :M] = torch.from_numpy(np.ascontiguousarray(X.T)).cuda()
    nb = K // 32
    Q = torch.zeros((nb, ld, 16), dtype=torch.uint8, device="cuda")
    S = torch.zeros((nb, ld), dtype=torch.uint8, device="cuda")
    tw.tw_quant_mx4(Xd.data_ptr(), M, K, ld, tw.LAYOUT_KM, Q.data_ptr(), S.data_ptr(), ld, _stream())
    codes, scale = ofb.mx4_quant(np.ascontiguousarray(X.T))
    assert np.array_equal(Q[:, :M].cpu().numpy(), ofb.mx4_bytes(codes))
    B, m = (rng.standard_normal((K, N)) * 0.05).astype(np.float16), np.ones((K, N), np.uint8)
    p = tw.tw_pack_mx4(B, m, G)
    C = torch.zeros((N, ld), dtype=torch.float16, device="cuda")
    tw.tw_gemm_mx4(Q.data_ptr(), S.data_ptr(), M, ld, p, C.data_ptr(), ld, _stream())
    fu.assert_mx4_close(C[:, :M].cpu().numpy(), codes, scale, B, m, G)
    del Q, S, C
    Q8 = torch.zeros((K, ld), dtype=torch.int8, device="cuda")
    s8 = torch.zeros((M,), device="cuda")
    tw.tw_quant_i8(Xd.data_ptr(), M, K, ld, Q8.data_ptr(), ld, s8.data_ptr(), _stream())
    assert np.array_equal(Q8[:, :M].cpu().numpy().T, ofb.quant_i8(X)[0])
