"""Few-bit operators without a GPU: the oracle's definitions against slower ones, the 4-bit packer against the oracle, and
every refusal of the entry points (nothing is launched: the checks come first)."""
import os
import shutil
import subprocess

import numpy as np
import pytest

import paper_2402_10876_amd as tw
from oracle import fewbit as ofb
from tests.fewbit_util import acts, block_mask
from tests.helpers import random_tvw_mask, random_tw_mask

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# ---- the oracle ------------------------------------------------------------------------------
def test_int8_rounding_is_the_exact_one():
    rng = np.random.default_rng(1)
    for top in (1.0, 3.0, 254.0, 0.333, 2.0 ** -24, 65504.0):
        top = float(np.float16(top))
        g = np.concatenate([(np.arange(-254, 255) / 254.0 * top).astype(np.float16),
                            (rng.uniform(-1, 1, 300) * top).astype(np.float16)]).astype(np.float64)
        g = np.append(g[np.abs(g) <= top], top)
        q, _ = ofb._quant(g[None], np.ones(1))
        assert q[0].tolist() == [ofb.round_ratio_exact(v, top) for v in g]
    assert ofb._quant(np.array([[0.5, 1.0, -0.5]]), np.ones(1))[0][0].tolist() == [64, 127, -64]     # 63.5 to even


def test_norm_definition_by_hand():
    X = np.array([[3.0, -4.0]], np.float16)
    h, y, q, s = ofb.rmsnorm(X, None, np.array([1.0, 2.0], np.float16), eps=12.5)
    assert np.array_equal(h, X) and np.allclose(y, [[0.6, -1.6]], rtol=1e-15)       # sqrt(12.5 + 12.5) = 5
    assert q.tolist() == [[48, -127]] and np.allclose(s, 8.0 / 5 / 127, rtol=1e-15)  # 127 * 3 / 8 = 47.6
    h, _, _, _ = ofb.rmsnorm(X, np.array([[2.0 ** -10, 1.0]], np.float16))
    assert h.tolist() == [[3.0, -3.0]]                                              # 3 + 2^-10 is a tie: to even


def test_mx4_definition_against_a_search():
    rng = np.random.default_rng(2)
    for i in range(60):
        n = int(rng.integers(1, 33))
        x = (rng.standard_normal(n) * 2.0 ** rng.integers(-20, 14)).astype(np.float16)
        x[rng.random(n) < 0.2] = 0
        if i % 3 == 0:
            x = (rng.integers(-16, 17, n) / 4.0).astype(np.float16)                 # ties
        codes, scale = ofb.mx4_quant(x[:, None])
        s, c = ofb.mx4_block(x)
        assert scale[0, 0] == s and codes[0, 0, :n].tolist() == c and not codes[0, 0, n:].any()
    s, c = ofb.mx4_block([5.0, 2.5, -7.5, 0.75, 0.25, 1.25, 3.5, 1.75])              # every tie, and past 6
    assert s == 127 and c == [6, 4, 15, 2, 0, 2, 6, 4]


def test_mx4_values_are_fp16_and_quantise_to_themselves():
    rng = np.random.default_rng(3)
    X = (rng.standard_normal((96, 200)) * 2.0 ** rng.integers(-24, 14, (1, 200))).astype(np.float16)
    X[:, 0] = (rng.integers(-7, 8, 96) * 2.0 ** -24).astype(np.float16)
    codes, scale = ofb.mx4_quant(X)
    V = ofb.mx4_values(codes, scale, 96)
    assert np.array_equal(V.astype(np.float16).astype(np.float64), V)
    again = ofb.mx4_quant(V.astype(np.float16))
    assert np.array_equal(again[0], codes) and np.array_equal(again[1], scale)


# ---- the packer ------------------------------------------------------------------------------
@pytest.mark.parametrize("seed", range(10))
def test_packed_values_and_mask_are_the_oracles(seed):
    rng = np.random.default_rng(seed)
    K, N, G = int(rng.integers(1, 200)), int(rng.integers(1, 300)), int(rng.choice([64, 128]))
    B = (rng.standard_normal((K, N)) * 2.0 ** rng.integers(-26, 13, (1, N))).astype(np.float16)
    mask = [lambda: block_mask(rng, K, N, G), lambda: random_tw_mask(rng, K, N, G),
            lambda: random_tvw_mask(rng, K, N, G)[0], lambda: (rng.random((K, N)) < 0.02).astype(np.uint8)][seed % 4]()
    B[mask == 0] = np.nan                                    # pruned weights are not looked at
    p = tw.tw_pack_mx4_host(B, mask, G)
    W, m = p.unpack()
    want = ofb.mx4_weight(B, mask).astype(np.float16)
    assert np.array_equal(W, want.view(np.uint16))
    cols, tiles = ofb.mx4_kept_rows(mask, G)
    keep = np.zeros((K, N), np.uint8)
    for t, rows in enumerate(tiles):
        keep[np.ix_(rows, cols[t * G:(t + 1) * G])] = 1
    assert np.array_equal(m, keep)
    e = p.export()
    assert e["dtype"] == tw.DTYPE_MX4 and np.array_equal(e["col_idx"], cols)
    assert p.flop_counts()[0] == keep.sum()
    q = tw.tw_pack_mx4_host(W.view(np.float16), m, G)         # a weight that is in the format already
    assert np.array_equal(q.unpack()[0], W)
    p.free()
    q.free()


def test_concatenation_keeps_the_members():
    rng = np.random.default_rng(5)
    K, G = 100, 64
    parts, Ws, ms = [], [], []
    for n, keep in ((70, 0.8), (64, 0.0), (130, 1.0)):        # the middle one keeps nothing
        mask = block_mask(rng, K, n, G, keep)
        B = rng.standard_normal((K, n)).astype(np.float16)
        parts.append(tw.tw_pack_mx4_host(B, mask, G))
        W, m = parts[-1].unpack()
        Ws.append(W)
        ms.append(m)
    c = tw.tw_concat(parts, upload=False)
    W, m = c.unpack()
    assert np.array_equal(W, np.concatenate(Ws, 1)) and np.array_equal(m, np.concatenate(ms, 1))
    i8 = tw.tw_pack_i8_host(np.ones((K, 64), np.int8), np.ones((K, 64), np.uint8), G)
    with pytest.raises(tw.TwError) as e:
        tw.tw_concat([parts[0], i8], upload=False)
    assert e.value.status == 1


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_packer_under_asan_ubsan(tmp_path):
    src = tmp_path / "driver.cpp"
    src.write_text(r"""
#include <cstdio>
#include <random>
#include <vector>
#include "mx4_format.h"
#include "packed.h"
int main() {
  std::mt19937 rng(7);
  int fails = 0;
  for (int h = 0; h < 0x7c00; ++h)                  // every finite magnitude: value of the code of the value
    for (int up = 0; up < 3; ++up) {
      const int top = std::min(h + 1024 * up, 0x7bff);
      const uint8_t s = twg::mx4_scale_of((uint16_t)top), c = twg::mx4_code((uint16_t)h, twg::mx4_factor(s));
      const uint16_t v = twg::mx4_value(c, s);
      if (twg::mx4_code(v, twg::mx4_factor(s)) != c || (up == 0 && twg::mx4_scale_of(v) != s)) ++fails;
    }
  for (int it = 0; it < 40; ++it) {
    const int K = 1 + rng() % 150, N = 1 + rng() % 300, G = rng() % 2 ? 64 : 128;
    std::vector<uint16_t> B((size_t)K * N);
    std::vector<uint8_t> mask((size_t)K * N);
    for (auto& b : B) { b = (uint16_t)rng(); if ((b & 0x7c00) == 0x7c00) b &= 0x83ff; }
    for (int b = 0; b < K; b += 32)
      for (int n = 0; n < N; ++n) {
        const bool keep = (n / 40 * 7 + b / 32) % 3 != 0 && n % 11 != 0;
        for (int k = b; k < std::min(K, b + 32); ++k) mask[(size_t)k * N + n] = keep;
      }
    tw_handle_s a, b, c;
    if (twg::pack_mx4_host(B.data(), mask.data(), K, N, G, &a) != TW_OK) { ++fails; continue; }
    if (twg::pack_mx4_host(B.data(), mask.data(), K, N, G, &b) != TW_OK) { ++fails; continue; }
    const tw_handle_s* parts[2] = {&a, &b};
    if (twg::concat_host(parts, 2, &c) != TW_OK) ++fails;
    if (c.mx4.vals.size() != 2 * a.mx4.vals.size() || c.mx4.n_members != 2) ++fails;
    std::vector<uint16_t> W((size_t)K * N);
    twg::unpack_host(&a, W.data(), nullptr);
    if (twg::pack_mx4_host(W.data(), mask.data(), K, N, G, &(b = tw_handle_s())) != TW_OK || b.mx4.vals != a.mx4.vals || b.mx4.scales != a.mx4.scales) ++fails;
  }
  std::printf("done fails=%d\n", fails);
  return fails ? 1 : 0;
}
""")
    exe = tmp_path / "driver"
    r = subprocess.run(["g++", "-std=c++17", "-g", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                        "-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(ROOT, "paper_2402_10876_amd", "csrc"), str(src),
                        os.path.join(ROOT, "paper_2402_10876_amd", "csrc", "pack.cpp"), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300, env=dict(os.environ, LD_PRELOAD=""))
    assert r.returncode == 0, r.stdout + r.stderr[-3000:]


# ---- refusals ----------------------------------------------------------------------------------
P = 0x10000        # never dereferenced


def _status(f, *a):
    with pytest.raises(tw.TwError) as e:
        f(*a)
    return e.value.status


def _each(f, good, changes, handle_ok=None):
    """Every change of one argument is refused with its status."""
    for i, v, st in changes:
        a = list(good)
        a[i] = v
        assert _status(f, *a) == st, (f.__name__, i, v)


def test_norm_and_int8_quantiser_refuse():
    #       X  R     gamma eps   M  K  ld H     Y     Q   ldq scale
    good = [P, 2 * P, P, 1e-6, 9, 5, 16, 3 * P, 4 * P, 5 * P, 16, P]
    _each(tw.tw_rmsnorm, good, [
        (0, None, 1), (0, P + 8, 1), (1, P + 2, 1), (1, None, 1), (2, P + 1, 1), (3, 0.0, 1), (3, -1.0, 1), (3, float("nan"), 1),
        (3, float("inf"), 1), (4, 0, 1), (4, -3, 1), (4, 17, 1), (5, 0, 1), (6, 8, 1), (6, 12, 1), (7, P + 8, 1), (8, P + 4, 1),
        (9, None, 1), (9, P + 4, 1), (10, 8, 1), (10, 24, 1), (11, None, 1), (11, P + 2, 1), (5, 131072, 3)])
    a = list(good)
    a[8] = a[9] = a[11] = None
    assert _status(tw.tw_rmsnorm, *a) == 1                     # no output
    a = list(good)
    a[4], a[6], a[10] = (1 << 27) + 1, (1 << 27) + 16, (1 << 27) + 16
    assert _status(tw.tw_rmsnorm, *a) == 3
    _each(tw.tw_quant_i8, [P, 9, 5, 16, P, 16, P], [
        (0, None, 1), (0, P + 2, 1), (1, 0, 1), (1, 17, 1), (2, 0, 1), (3, 12, 1), (4, None, 1), (4, P + 8, 1), (5, 8, 1), (5, 20, 1),
        (6, None, 1), (6, P + 1, 1), (2, 131072, 3)])


def test_an_output_that_is_another_operand_is_refused():
    #       X  R     gamma  eps   M  K  ld H     Y      Q    ldq scale
    good = [P, 2 * P, 3 * P, 1e-6, 9, 5, 16, 4 * P, 5 * P, 6 * P, 16, 7 * P]
    for out in (8, 9, 11):
        _each(tw.tw_rmsnorm, good, [(out, good[i], 1) for i in (0, 1, 2, 7, 8, 9, 11) if i != out])
    _each(tw.tw_rmsnorm, good, [(7, good[2], 1)])
    _each(tw.tw_quant_i8, [P, 9, 5, 16, 2 * P, 16, 3 * P], [(4, P, 1), (6, P, 1), (6, 2 * P, 1)])
    for layout in (tw.LAYOUT_KM, tw.LAYOUT_MK):
        _each(tw.tw_quant_mx4, [P, 9, 5, 16, layout, 2 * P, 3 * P, 16], [(5, P, 1), (6, P, 1), (6, 2 * P, 1)])


def test_mx4_calls_refuse():
    _each(tw.tw_quant_mx4, [P, 9, 5, 16, tw.LAYOUT_KM, P, P, 16], [
        (0, None, 1), (0, P + 8, 1), (1, 0, 1), (2, 0, 1), (3, 8, 1), (3, 20, 1), (4, 2, 1), (5, None, 1), (5, P + 8, 1),
        (6, None, 1), (6, P + 8, 1), (7, 8, 1), (7, 24, 1), (2, 131072, 3), (7, (1 << 27) + 16, 3)])
    _each(tw.tw_quant_mx4, [P, 9, 30, 32, tw.LAYOUT_MK, P, P, 16], [(3, 24, 1), (3, 34, 1)])
    B, one = np.ones((40, 70), np.float16), np.ones((40, 70), np.uint8)
    assert _status(tw.tw_pack_mx4_host, B, one, 32) == 3 and _status(tw.tw_pack_mx4_host, B, one, 100) == 1
    assert _status(tw.tw_pack_mx4_host, np.ones((131072, 1), np.float16), np.ones((131072, 1), np.uint8), 64) == 3
    for bad in (np.inf, -np.inf, np.nan):
        B2 = B.copy()
        B2[33, 69] = bad
        assert _status(tw.tw_pack_mx4_host, B2, one, 64) == 1
    with pytest.raises(TypeError):
        tw.tw_pack_mx4_host(B.astype(np.float32), one, 64)
    with pytest.raises(ValueError):
        tw.tw_pack_mx4_host(B, one[:, :5], 64)
    w = tw.tw_pack_mx4_host(B, one, 64)
    two = tw.tw_concat([w, tw.tw_pack_mx4_host(B[:, :5], one[:, :5], 64)], upload=False)
    f16 = tw.tw_pack_host(B, one, 64, tw.PATTERN_TW)
    i8 = tw.tw_pack_i8_host(np.ones((40, 70), np.int8), one, 64)
    _each(tw.tw_gemm_mx4, [P, P, 9, 16, w, P, 16], [
        (0, None, 1), (0, P + 8, 1), (1, None, 1), (1, P + 8, 1), (2, 0, 1), (2, 17, 1), (3, 8, 1), (3, 24, 1), (5, None, 1),
        (5, P + 8, 1), (6, 8, 1), (6, 20, 1), (4, f16, 1), (4, i8, 1)])
    assert _status(tw.tw_gemm_mx4, P, P, 9, 16, w, P, 16) == 6                       # not uploaded
    _each(tw.tw_gemm_mx4_grouped, [P, P, 9, 16, P, w, P, 16], [
        (0, None, 1), (4, None, 1), (4, P + 2, 1), (5, f16, 1), (5, two, 1), (6, None, 1), (7, 8, 1), (2, 0, 1)])
    assert _status(tw.tw_gemm_mx4_grouped, P, P, 9, 16, P, w, P, 16) == 6
    # the other products do not take the handle
    assert _status(tw.tw_gemm, P, 8, 8, tw.LAYOUT_KM, w, P, 8) == 1
    assert _status(tw.tw_gemm_i8, P, 16, 16, w, P, 16) == 1
    assert _status(tw.tw_gemm_i8_scaled, P, 16, 16, w, P, P, P, 16) == 1

    class G:
        C, R, S, B, H, W, P, L = 40, 1, 1, 1, 2, 2, 2, 2
    assert _status(tw.tw_conv_bind, w, G, 8) == 3
    w.free()
    with pytest.raises(ValueError):
        tw.tw_gemm_mx4(P, P, 9, 16, w, P, 16)


def test_scaled_int8_product_refuses():
    one = np.ones((40, 70), np.uint8)
    w = tw.tw_pack_i8_host(np.ones((40, 70), np.int8), one, 64)
    f16 = tw.tw_pack_host(np.ones((40, 70), np.float16), one, 64, tw.PATTERN_TW)
    _each(tw.tw_gemm_i8_scaled, [P, 9, 16, w, P, P, P, 16], [
        (0, None, 1), (0, P + 4, 1), (1, 0, 1), (1, 17, 1), (2, 8, 1), (2, 24, 1), (3, f16, 1), (4, None, 1), (4, P + 2, 1),
        (5, None, 1), (5, P + 2, 1), (6, None, 1), (6, P + 8, 1), (7, 8, 1), (7, 20, 1)])
    assert _status(tw.tw_gemm_i8_scaled, P, 9, 16, w, P, P, P, 16) == 6


def test_launch_calls_through_the_module_end_as_with_ctypes():
    """Each argument in turn as an odd object: the same refusal or conversion on both routes (nothing is launched: the
    weights are not uploaded and the calls without one get an invalid size)."""
    from paper_2402_10876_amd import binding
    tw.lib()
    assert binding._call is not binding._Unbound
    one = np.ones((40, 70), np.uint8)
    w4 = tw.tw_pack_mx4_host(np.ones((40, 70), np.float16), one, 64)
    w8 = tw.tw_pack_i8_host(np.ones((40, 70), np.int8), one, 64)
    calls = [(tw.tw_rmsnorm, [P, P, P, 1e-6, 0, 5, 16, P, P, P, 16, P, 0]), (tw.tw_quant_i8, [P, 0, 5, 16, P, 16, P, 0]),
             (tw.tw_quant_mx4, [P, 0, 5, 16, 0, P, P, 16, 0]), (tw.tw_gemm_i8_scaled, [P, 9, 16, w8, P, P, P, 16, 0]),
             (tw.tw_gemm_mx4, [P, P, 9, 16, w4, P, 16, 0]), (tw.tw_gemm_mx4_grouped, [P, P, 9, 16, P, w4, P, 16, 0])]

    def outcome(f, a):
        try:
            return f(*a)
        except Exception as e:
            return type(e), getattr(e, "status", None)
    for f, good in calls:
        for i, v in enumerate(good):
            if v is w4 or v is w8:
                continue
            if i == {tw.tw_rmsnorm: 4, tw.tw_quant_i8: 1, tw.tw_quant_mx4: 1}.get(f):
                odds = [v, None, True and 0, 0.0, "8", -1, 1 << 40]        # stays a size that is refused
            else:
                odds = [v, None, True, 8.0, "8", np.int64(8), -1, 1 << 31, 1 << 64]
            for o in odds:
                a = list(good)
                a[i] = o
                got = outcome(f, a)
                call, binding._call = binding._call, binding._Unbound
                try:
                    want = outcome(f, a)
                finally:
                    binding._call = call
                assert got == want, (f.__name__, i, o)
    m = binding._call
    assert m.rmsnorm(1) is None and m.quant_mx4(0, 1) is None and m.gemm_mx4(0, 0, 1, 16, None, 0, 8, 0) is None


def test_row_count_check_of_the_masked_definition():
    """acts() holds what its users rely on."""
    x = acts(1, 9, 50)
    assert not x[4].any() and np.abs(x[8]).max() < 2.0 ** -14
