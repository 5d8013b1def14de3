"""Few-bit operators at the ends of what they allow: factors of the norm that are not finite, the most values of a
row-major quantiser, every number of tokens of an int8 output, 4-bit products where the shape of the tiles changes
(-m gpu)."""
import numpy as np
import pytest

import paper_2402_10876_amd as tw
from oracle import fewbit as ofb
from oracle import gemm as og
from tests import fewbit_util as fu
from tests.fewbit_util import acts, up
from tests.helpers import random_tw_mask
import workloads as wl

pytestmark = pytest.mark.gpu


def _norm(X, R, gamma, eps, i8, f16):
    """h, y, int8 values (tokens first) and scales of one call, the columns behind M looked at."""
    import torch
    M, K = X.shape
    ld, ldq = up(M, 8), up(M, 16)
    new = lambda shape, fill, dtype: torch.full(shape, fill, dtype=dtype, device="cuda")  # noqa: E731
    Xd, Rd = fu.dev_km(X, ld), None if R is None else fu.dev_km(R, ld)
    gd = None if gamma is None else torch.from_numpy(gamma).cuda()
    H = None if R is None else new((K, ld), 7.0, torch.float16)
    Y = new((K, ld), 7.0, torch.float16) if f16 else None
    Q = new((K, ldq), 99, torch.int8) if i8 else None
    s = new((M,), 7.0, torch.float32) if i8 else None
    p = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    tw.tw_rmsnorm(p(Xd), p(Rd), p(gd), eps, M, K, ld, p(H), p(Y), p(Q), ldq, p(s), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    out = []
    for t, fill in ((H, 7.0), (Y, 7.0), (Q, 99)):
        if t is not None:
            assert bool((t[:, M:] == fill).all())
        out.append(None if t is None else t[:, :M].cpu().numpy().T)
    return (*out, None if s is None else s.cpu().numpy())


def _assert_y(got, y, K):
    """got: fp16 output, y: fp64 definition (NaN and infinities among them): NaN and each infinity in their places, every
    other value within the roundings of fu.norm_tol and half a step of fp16."""
    got = got.astype(np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(y))
    inf = np.isinf(y)
    assert np.array_equal(got[inf], y[inf])
    fine = np.isfinite(y)
    assert np.isfinite(got[fine]).all()
    err, size = np.abs(got[fine] - y[fine]), np.abs(y[fine])
    assert (err <= size * (fu.STEP16 + fu.norm_tol(K)) * (1 + fu.STEP16) + 2.0 ** -25).all()


# One launch that keeps its rows, one that reads them again (2050 rows of 4100, 8200 and 16384 tokens without a residual), slices.
@pytest.mark.parametrize("M,K,residual", [(1, 1, False), (40, 5, True), (40, 1500, False), (33, 1003, True), (3000, 700, True),
                                          (4100, 300, False), (4100, 2050, False), (8200, 2050, False), (16384, 2049, False), (16400, 2049, False), (24001, 2050, False), (16450, 96, True),
                                          (70, 4200, True), (1030, 2100, True), (100, 6000, False), (3, 8200, False), (5, 8200, True)])
@pytest.mark.parametrize("i8,f16", [(False, True), (True, True), (True, False)])
def test_norm_with_factors_that_are_not_finite(M, K, residual, i8, f16):
    """Every token's scale is NaN and its int8 values are 0; the fp16 output is the formula's, whose root-mean-square does
    not contain the factors: only their own rows (and a token that is not finite itself) hold infinities and NaN."""
    X = acts(M + K, M, K)
    R = acts(M + K + 1, M, K, 3.0) if residual else None
    if M > 6:
        X[5, K // 3] = -np.inf
    for bads in ([np.inf, -np.inf, np.nan], [np.nan], [np.inf], [-np.inf])[:4 if M * K < 1 << 22 else 1]:
        gamma = (1 + 0.3 * np.random.default_rng(K).standard_normal(K)).astype(np.float16)
        at = [(K // 2 + 131 * i) % K for i in range(len(bads))]
        for k, bad in zip(at, bads):
            gamma[k] = bad
        print(f"norm M={M} K={K} residual={residual} i8={i8} f16={f16} gamma={bads}", flush=True)
        h, y, q, scale = ofb.rmsnorm(X, R, gamma, 1e-5)
        assert np.isnan(scale).all() and not q.any()
        if M > 6 and K > 3:
            assert np.isfinite(np.delete(np.delete(y, 5, 0), at, 1)).all()
        H, Y, Q, s = _norm(X, R, gamma, 1e-5, i8, f16)
        if H is not None:
            assert np.array_equal(H.view(np.uint16), h.view(np.uint16))
        if Y is not None:
            _assert_y(Y, y, K)
        if Q is not None:
            assert not Q.any() and np.isnan(s).all()

def test_row_major_quantiser_of_the_most_tokens():
    """2^27 row-major tokens of 520 values: more threads than one dimension of a grid takes."""
    import torch
    M, K, ldx, nb = 1 << 27, 520, 520, 17
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 190 << 30:
        pytest.skip("needs 170 GiB of device memory")
    dev = "cuda"
    X = torch.zeros((M, ldx), dtype=torch.float16, device=dev)
    Q = torch.full((nb, M, 16), 0xA5, dtype=torch.uint8, device=dev)
    S = torch.full((nb, M), 0xA5, dtype=torch.uint8, device=dev)
    rows = np.unique(np.concatenate([np.arange(20), (1 << 26) + np.arange(-17, 18), M - 1 - np.arange(40),
                                     np.random.default_rng(1).integers(0, M, 200)]))
    x = acts(4, rows.size, K)
    at = torch.from_numpy(rows).to(dev)
    X[at] = torch.from_numpy(x).to(dev)
    print("row-major quantiser, 2^27 tokens of 520 values", flush=True)
    tw.tw_quant_mx4(X.data_ptr(), M, K, ldx, tw.LAYOUT_MK, Q.data_ptr(), S.data_ptr(), M, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    codes, scale = ofb.mx4_quant(np.ascontiguousarray(x.T))
    assert np.array_equal(Q[:, at].cpu().numpy(), ofb.mx4_bytes(codes))
    assert np.array_equal(S[:, at].cpu().numpy(), scale)
    for b in range(nb):                              # every other token is zeros
        S[b, at] = 127
        assert bool((S[b] == 127).all())
        Q[b, at] = 0
        assert not bool(Q[b].any())
    del X, Q, S
    torch.cuda.empty_cache()


@pytest.mark.parametrize("tile_m", [64, 128, 256])
def test_int8_output_of_any_number_of_tokens(tile_m):
    """The last piece of 16 tokens of a column holds 1 to 16 of them, for every height of the tiles and for weights of both
    widths of tiles; the columns behind M are left as they were."""
    import torch
    rng = np.random.default_rng(5)
    K, N = 140, 150
    B = wl.rng_i8(K, (K, N))
    for G in (64, 128):
        mask = random_tw_mask(rng, K, N, G)
        p = tw.tw_pack_i8(B, mask, G, tw.PATTERN_TW)
        for M in range(497, 514):
            A, ld = wl.rng_i8(M, (M, K)), up(M, 16) + 16
            At = np.full((K, ld), 0x55, np.int8)
            At[:, :M] = A.T
            Ad = torch.from_numpy(At).cuda()
            C = torch.full((N, ld), 99, dtype=torch.int8, device="cuda")
            print(f"int8 output tile_m={tile_m} G={G} M={M}", flush=True)
            tw.tw_set_option("tile_m", tile_m)
            try:
                tw.tw_gemm_i8(Ad.data_ptr(), M, ld, p, C.data_ptr(), ld, 1, 1e-3, torch.cuda.current_stream().cuda_stream)
            finally:
                tw.tw_set_option("tile_m", 0)
            got = C.cpu().numpy()
            sums = np.rint(A.astype(np.float64) @ (B * (mask != 0)).astype(np.float64))
            assert np.array_equal(got[:, :M].T, og.requantize_i8(sums.astype(np.int64), 1e-3))
            assert (got[:, M:] == 99).all()
        p.free()


def _mx4(M, K, N, G, off=None):
    """Products of 4-bit operands against the definition; off: the first tokens of every expert (the same weight for all)."""
    import torch
    rng = np.random.default_rng(M + K + N)
    mask = fu.block_mask(rng, K, N, G, 0.95, 0.9)
    B = (rng.standard_normal((K, N)) * 0.05).astype(np.float16)
    X = acts(M, M, K)
    X[M - 2, K // 3] = np.inf
    stream = torch.cuda.current_stream().cuda_stream
    Q, S = fu.quant_mx4_dev(tw, X, tw.LAYOUT_MK, stream)
    p = tw.tw_pack_mx4(B, mask, G)
    h = p if off is None else tw.tw_concat([p] * (len(off) - 1))
    ldc = up(M, 8) + 8
    C = torch.full((N, ldc), 7.0, dtype=torch.float16, device="cuda")
    print(f"4-bit product M={M} K={K} N={N} G={G} off={off}", flush=True)
    if off is None:
        tw.tw_gemm_mx4(Q.data_ptr(), S.data_ptr(), M, Q.shape[1], h, C.data_ptr(), ldc, stream)
    else:
        o = torch.tensor(off, dtype=torch.int32, device="cuda")
        tw.tw_gemm_mx4_grouped(Q.data_ptr(), S.data_ptr(), M, Q.shape[1], o.data_ptr(), h, C.data_ptr(), ldc, stream)
    torch.cuda.synchronize()
    got = C.cpu().numpy()
    a, b = (0, M) if off is None else (off[0], off[-1])
    assert (got[:, :a] == 7).all() and (got[:, b:] == 7).all()
    codes, scale = ofb.mx4_quant(np.ascontiguousarray(X.T))
    fu.assert_mx4_close(got[:, a:b], codes[:, a:b], scale[:, a:b], B, mask, G)


@pytest.mark.parametrize("M,K,N,G", [
    (1000, 500, 1000, 128), (1500, 500, 1000, 128), (900, 200, 1000, 128), (1300, 200, 1000, 128),      # short lists: shared or single waves
    (1000, 2000, 1000, 128), (1150, 2000, 1000, 64), (3000, 300, 500, 64), (5000, 300, 500, 64),        # long ones; pairs of waves
    (3100, 2100, 4000, 128), (8199, 1030, 2200, 128), (12001, 1030, 2200, 128), (5400, 2100, 4000, 128),  # one round, one barely begun, more
    (700, 1100, 4000, 128), (900, 1100, 4000, 128), (700, 2100, 4000, 128), (1090, 1100, 4000, 128), (1090, 2100, 4000, 128),
    (4700, 500, 1000, 128)])
def test_4_bit_products_where_tile_shapes_change(M, K, N, G):
    _mx4(M, K, N, G)


@pytest.mark.parametrize("K,N,G,off", [
    (500, 1000, 128, [0, 100, 100, 350, 600, 610, 700, 790, 803]), (500, 1000, 128, [1, 300, 301, 700, 1201]),
    (300, 500, 64, [0, 700, 1500, 1501, 3001]), (1100, 1000, 128, [0, 1000, 2500, 2501, 5000, 6000, 7700, 8000, 9000]),
    (300, 2000, 128, [5, 1300, 2600, 3900, 5301]), (1030, 2200, 128, [5, 6001, 12010])])
def test_4_bit_products_by_expert_where_tile_shapes_change(K, N, G, off):
    _mx4(off[-1] + 3, K, N, G, off)
