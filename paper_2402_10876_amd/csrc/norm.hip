// Root-mean-square norm with the residual's addition, output in int8 with a scale per token and / or in fp16, and the int8
// quantiser alone.  K x M activations: a token is a column, its K values ld elements apart.
//
//   h = fp16(x + r);  g = h * gamma (exact in fp32: two 11-bit mantissas);  inv = 1 / sqrt(mean h^2 + eps)
//   y = fp16(g * inv);  scale = max |g| * inv / 127;  q = nearest integer of 127 g / max |g|, ties to even
//
// inv cancels in q, which is therefore exact: u = fma(g, fl(127 / max|g|), 1.5 * 2^23) rounds to an integer in the low byte of
// u, wrong only within 127 * 2^-24 of a half; where the distance to n is more than 0.49998 the side is settled in 64 bits
// (254 g against (2n +- 1) max|g|, both exact).  Sums of squares are fp32: at most ceil(K / 128)
// terms in a row, then a tree and 16 waves.
//
// Bound by memory: 2 bytes in per value (4 with a residual), 1 to 5 out.  One workgroup owns 8 to 64 tokens and all K rows and
// keeps its values in registers (and LDS) between the two passes, up to 16 rows a lane; longer columns are read again, from L2.
// Tokens of more than 8192 rows go in slices of their rows (below), shorter ones where that was measured to be faster, the int8
// quantiser's as well as the norm's (slices_pay).
#include <type_traits>

#include "device_common.h"
#include "fewbit.h"

namespace twg {

namespace {

constexpr float MAGIC = 12582912.f;      // 1.5 * 2^23
constexpr uint32_t INF_BITS = 0x7f800000u;

// The integer nearest to 127 g / top where n is next to a half away (d: which side).
__device__ __forceinline__ float settle(float g, float top, float n, float d) {
  const double sgn = d > 0.f ? 1.0 : -1.0;
  const double x = 254.0 * (double)g, edge = (2.0 * (double)n + sgn) * (double)top;
  const bool odd = ((int)n & 1) != 0;
  if (d > 0.f) return (x > edge || (x == edge && odd)) ? n + 1.f : n;
  return (x < edge || (x == edge && odd)) ? n - 1.f : n;
}

// What a token is finished with, from its sum of squares and its largest |g| (INF_BITS: not finite).
struct Token { float inv, top, mul, scale; };
template <bool NORM>
__device__ __forceinline__ Token finish_token(float sum, uint32_t top, const NormArgs& g) {
  Token t;
  t.inv = 1.f;
  if constexpr (NORM) t.inv = 1.f / sqrtf(sum / (float)g.K + g.eps);
  const bool fine = top != 0 && top < INF_BITS;
  t.top = __uint_as_float(top);
  t.mul = fine ? 127.f / t.top : 0.f;
  t.scale = fine ? t.top * t.inv / 127.f : top == 0 ? 0.f : __builtin_nanf("");
  return t;
}

// Eight tokens of a row to int8 (top: of these tokens, in LDS).
__device__ __forceinline__ uint2 round8(const float (&f)[8], const float (&mul)[8], const float* top) {
  float u[8], d[8], far = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    u[e] = __builtin_fmaf(f[e], mul[e], MAGIC);
    d[e] = __builtin_fmaf(f[e], mul[e], MAGIC - u[e]);
    far = __builtin_fmaxf(far, __builtin_fabsf(d[e]));
  }
  if (far > 0.49998f) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (__builtin_fabsf(d[e]) > 0.49998f) u[e] = settle(f[e], top[e], u[e] - MAGIC, d[e]) + MAGIC;
  }
  uint32_t q[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(u[4 * e + 1]), __float_as_uint(u[4 * e]), 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(u[4 * e + 3]), __float_as_uint(u[4 * e + 2]), 0x04000c0cu);
    q[e] = lo | hi;
  }
  return make_uint2(q[0], q[1]);
}
// Eight tokens of a row to memory; only the first `tail` of the piece that ends behind the last token, in stores of 4, 2 and 1
// (one by one they made the workgroup of that piece the last: int8 quantiser, 1003 rows, 1957 tokens 7.2 us, 1968 tokens 5.6).
__device__ __forceinline__ void store8(_Float16* p, half8 v, bool whole, int tail) {
  if (whole) *(half8*)p = v;
  else store_front(p, v, tail);
}
__device__ __forceinline__ void store8(int8_t* p, uint2 q, bool whole, int tail) {
  if (whole) {
    *(uint2*)p = q;
    return;
  }
  uint32_t a = q.x;
  if (tail & 4) {
    *(uint32_t*)p = a;
    a = q.y;
  }
  if (tail & 2) {
    *(uint16_t*)(p + (tail & 4)) = (uint16_t)a;
    a >>= 16;
  }
  if (tail & 1) p[tail & 6] = (int8_t)a;
}

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(ushort2v, a), __builtin_bit_cast(ushort2v, b)));
}

// Workgroup -> its first token.  The workgroups of a line of memory (64 tokens) run on one XCD, whose L2 then fetches it once.
// An XCD owns every other line of a quarter of the row: with all lines of an eighth, rows of a power of two of bytes meet half
// of its L2's channels or fewer.
constexpr int lines_of(int64_t M) { return (int)((M + 63) / 64); }
template <int TOK>
__device__ __forceinline__ int first_token(int bid, int n_wg) {
  constexpr int WPL = 64 / TOK;
  const int xcd = bid & 7, slot = bid >> 3, per = n_wg / (8 * WPL);
  const int line = (xcd >> 1) * 2 * per + slot / WPL * 2 + (xcd & 1);
  return line * 64 + slot % WPL * TOK;
}

// Eight values of a lane over the four rows of 16 lanes: x[0], x[1] of row r become the results for values 2 (r % 2) +
// 4 (r / 2) and the next.
template <class F>
__device__ __forceinline__ void halve(float (&x)[8], F f) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const auto v = __builtin_amdgcn_permlane32_swap(__float_as_uint(x[e]), __float_as_uint(x[e + 4]), false, false);
    x[e] = f(__uint_as_float(v[0]), __uint_as_float(v[1]));
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const auto v = __builtin_amdgcn_permlane16_swap(__float_as_uint(x[e]), __float_as_uint(x[e + 2]), false, false);
    x[e] = f(__uint_as_float(v[0]), __uint_as_float(v[1]));
  }
}
// Over the lanes of a row of 16 that are LPR apart.
template <int LPR, class F>
__device__ __forceinline__ float around(float x, F f) {
  auto turn = [&](auto N) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x120 + decltype(N)::value, 0xf, 0xf, true));
  };
  x = f(x, turn(std::integral_constant<int, 8>{}));
  if constexpr (LPR < 8) x = f(x, turn(std::integral_constant<int, 4>{}));
  if constexpr (LPR < 4) x = f(x, turn(std::integral_constant<int, 2>{}));
  if constexpr (LPR < 2) x = f(x, turn(std::integral_constant<int, 1>{}));
  return x;
}

}  // namespace

// TOK tokens and NT threads per workgroup; a lane keeps NCH rows in registers and NL in LDS (NCH = 0: more than fit, the
// second pass reads them again).
template <bool NORM, int TOK, int NT, int NCH, int NL = 0>
__global__ __launch_bounds__(NT) void norm_kernel(NormArgs g) {
  constexpr int LPR = TOK / 8;           // lanes per row, 8 tokens each
  constexpr int RPP = NT / LPR;          // rows per pass
  constexpr int NW = NT / 64;
  __shared__ half8 s_h[NL ? NL : 1][NL ? NT : 1];
  __shared__ __attribute__((aligned(16))) float s_sum[NW][TOK];
  __shared__ __attribute__((aligned(16))) uint32_t s_top[NW][TOK];
  __shared__ __attribute__((aligned(16))) float s_inv[TOK], s_mul[TOK], s_max[TOK];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int m0 = first_token<TOK>(blockIdx.x, gridDim.x);
  if (m0 >= g.M) return;
  const int c = tid % LPR, r0 = tid / LPR;
  const int m = m0 + c * 8;
  const bool live = m < g.M;
  const uint64_t lane_at = ((uint64_t)r0 * g.ld + (live ? c * 8 : 0)) * 2;   // bytes from row i * RPP, token m0
  const bool whole = m + 8 <= g.M;
  const int tail = g.M & 7;              // tokens of the one piece that is not
  const int n_ch = (g.K + RPP - 1) / RPP;

  // Rows r0 + (i0 + i) * RPP, i < N: values (rows behind K: zeros) and gammas.  Every kind of load or store is a loop of its
  // own behind one uniform branch, so that all of a kind are under way at once.
  auto load_x = [&](const _Float16* from, int i) {      // (lanes behind K: a row in front of it)
    const int k = i * RPP;
    const char* row = (const char*)(from + (size_t)(k < g.K ? k : 0) * g.ld + m0);
    return *(const half8*)(row + (r0 + k < g.K ? lane_at : 0));
  };
  auto load_h = [&](int i0, auto& h) {
    constexpr int N = sizeof(h) / sizeof(half8), B = N < 8 ? N : N == 8 ? 8 : 4;
#pragma unroll
    for (int i = 0; i < N; ++i) h[i] = load_x(g.X, i0 + i);
    if (NORM && g.R) {
#pragma unroll
      for (int b = 0; b < N; b += B) {
        half8 r[B];
#pragma unroll
        for (int i = 0; i < B; ++i) r[i] = load_x(g.R, i0 + b + i);
#pragma unroll
        for (int i = 0; i < B; ++i) h[b + i] += r[i];
        __builtin_amdgcn_sched_barrier(0);
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (r0 + (i0 + i) * RPP >= g.K) h[i] = half8{0, 0, 0, 0, 0, 0, 0, 0};
  };
  auto load_gamma = [&](int i0, auto& gam) {
    constexpr int N = sizeof(gam) / sizeof(_Float16);
#pragma unroll
    for (int i = 0; i < N; ++i) gam[i] = (_Float16)1.f;
    if (NORM && g.gamma) {
#pragma unroll
      for (int i = 0; i < N; ++i) gam[i] = g.gamma[min(r0 + (i0 + i) * RPP, g.K - 1)];
    }
  };
  auto store_half = [&](_Float16* to, int i, half8 v) {
    const int k = r0 + i * RPP;
    if (k < g.K && live) store8((_Float16*)((char*)(to + (size_t)(i * RPP) * g.ld + m0) + lane_at), v, whole, tail);
  };

  // Norm: sums of squares and the largest |g|, as fp32; an infinity or NaN among the h of a token shows in its sum, one
  // among the gamma in every token's largest |g| (not in the sums: Y is the formula's, whose inv does not contain gamma).
  // Quantiser: the largest magnitude over the fp16 bits.
  float sum[NORM ? 8 : 1], top[NORM ? 8 : 1], worst = 0.f;
  uint32_t bits[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int e = 0; e < (NORM ? 8 : 1); ++e) { sum[e] = 0.f; top[e] = 0.f; }
  auto stats = [&](half8 h, float gam) {
    if constexpr (NORM) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float f = (float)h[e];
        sum[e] = __builtin_fmaf(f, f, sum[e]);
        top[e] = __builtin_fmaxf(top[e], __builtin_fabsf(f * gam));
      }
      worst = __builtin_fmaf(gam, 0.f, worst);         // NaN once a gamma is not finite
    } else {
      const u32x4 v = __builtin_bit_cast(u32x4, h);
#pragma unroll
      for (int e = 0; e < 4; ++e) bits[e] = max_u16x2(bits[e], v[e] & 0x7fff7fffu);
    }
  };

  constexpr int NG = NCH ? NCH : 4;      // rows of a lane that are held at a time
  half8 h[NG];
  _Float16 gam[NG];
  auto first_pass = [&](int i0) {
    load_gamma(i0, gam);
    load_h(i0, h);
    if (NORM && g.H) {
#pragma unroll
      for (int i = 0; i < NG; ++i) store_half(g.H, i0 + i, h[i]);
    }
#pragma unroll
    for (int i = 0; i < NG; ++i) stats(h[i], (float)gam[i]);
  };
  if constexpr (NL > 0) {
    static_assert(NL <= NCH, "");
    first_pass(NCH);
#pragma unroll
    for (int i = 0; i < NL; ++i) s_h[i][tid] = h[i];
  }
  if constexpr (NCH > 0) first_pass(0);
  else
    for (int i0 = 0; i0 < n_ch; i0 += NG) first_pass(i0);

  // Over the lanes with the same tokens: two swaps between rows of 16 lanes halve the values of a lane (row r keeps tokens
  // 2 (r % 2) + 4 (r / 2) and the next one of its piece), then rotations inside the row; no LDS instruction (with
  // shuffles, 102 a wave, one token of 4096 values took 9 us, with these 5.6).
  const int tok = c * 8 + 2 * (lane >> 4 & 1) + 4 * (lane >> 5);
  if constexpr (NORM) {
#pragma unroll
    for (int e = 0; e < 8; ++e) top[e] = worst == 0.f ? top[e] : __builtin_inff();
    halve(sum, [](float x, float y) { return x + y; });
    halve(top, [](float x, float y) { return __builtin_fmaxf(x, y); });
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      sum[e] = around<LPR>(sum[e], [](float x, float y) { return x + y; });
      top[e] = around<LPR>(top[e], [](float x, float y) { return __builtin_fmaxf(x, y); });
    }
    if ((lane & 15) < LPR)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        s_sum[wave][tok + e] = sum[e];
        s_top[wave][tok + e] = sum[e] < __builtin_inff() ? __float_as_uint(top[e]) : INF_BITS;
      }
  } else {
    float t8[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t b = bits[e >> 1] >> (16 * (e & 1)) & 0xffffu;
      t8[e] = __uint_as_float(b);        // (ordered as floats of 2^-126 and less: the comparison below is one of integers)
    }
    auto most = [](float x, float y) { return __uint_as_float(max(__float_as_uint(x), __float_as_uint(y))); };
    halve(t8, most);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const uint32_t b = __float_as_uint(around<LPR>(t8[e], most));
      if ((lane & 15) < LPR)
        s_top[wave][tok + e] = b >= 0x7c00u ? INF_BITS : __float_as_uint((float)__builtin_bit_cast(_Float16, (unsigned short)b));
    }
  }
  __syncthreads();
  if (tid < TOK) {
    float s = 0.f;
    uint32_t t = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      if constexpr (NORM) s += s_sum[w][tid];
      t = max(t, s_top[w][tid]);
    }
    const Token x = finish_token<NORM>(s, t, g);
    s_inv[tid] = x.inv;
    s_max[tid] = x.top;
    s_mul[tid] = x.mul;
    if (g.scale && m0 + tid < g.M) g.scale[m0 + tid] = x.scale;
  }
  __syncthreads();
  float inv[8], mul[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) { inv[e] = s_inv[c * 8 + e]; mul[e] = s_mul[c * 8 + e]; }

  auto store_y = [&](int i, half8 x, float gm) {
    half8 y;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = (_Float16)((float)x[e] * gm * inv[e]);
    store_half(g.Y, i, y);
  };
  auto store_q = [&](int i, half8 x, float gm) {
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = NORM ? (float)x[e] * gm : (float)x[e];
    const uint2 q = round8(f, mul, s_max + c * 8);
    const int k = r0 + i * RPP;
    if (k < g.K && live) store8(g.Q + (size_t)(i * RPP) * g.ldq + m0 + ((uint64_t)r0 * g.ldq + c * 8), q, whole, tail);
  };
  auto second_pass = [&](int i0) {
    if (NORM && g.Y) {
#pragma unroll
      for (int i = 0; i < NG; ++i) store_y(i0 + i, h[i], (float)gam[i]);
    }
    if (g.Q) {
#pragma unroll
      for (int i = 0; i < NG; ++i) store_q(i0 + i, h[i], (float)gam[i]);
    }
  };
  if constexpr (NCH > 0) {
    if constexpr (NCH > 8) load_gamma(0, gam);
    second_pass(0);
    if constexpr (NL > 0) {
      load_gamma(NCH, gam);
#pragma unroll
      for (int i = 0; i < NL; ++i) h[i] = s_h[i][tid];
#pragma unroll
      for (int i = NL; i < NCH; ++i) h[i] = half8{0, 0, 0, 0, 0, 0, 0, 0};      // (rows behind K)
      second_pass(NCH);
    }
  } else
    for (int i0 = 0; i0 < n_ch; i0 += NG) {
      load_gamma(i0, gam);
      if (NORM && g.H) {                 // this lane's own stores (X or R may be the same buffer, and are gone then)
#pragma unroll
        for (int i = 0; i < NG; ++i) h[i] = load_x(g.H, i0 + i);
      } else {
        load_h(i0, h);
      }
      second_pass(i0);
    }
}

template <bool NORM, int TOK, int NT, int NCH, int NL = 0>
hipError_t run_norm(const NormArgs& g, hipStream_t stream) {
  const int per = (lines_of(g.M) + 7) / 8;
  return launch_kernel(norm_kernel<NORM, TOK, NT, NCH, NL>, dim3(8 * per * (64 / TOK)), dim3(NT), stream, g);
}

// ---- long tokens in slices of their rows ----------------------------------------------------------
// A workgroup that owns whole tokens reads and writes narrow pieces of rows (64 and 32 bytes, of lines of 128), and few tokens are
// few workgroups.  With long tokens three launches on 128 tokens x one slice of the rows are faster, every access whole lines: sums of
// the slices (and H), sums of the tokens, outputs.  No memory beyond the outputs is used: between the launches the sums of a slice,
// 8 bytes per token, lie in the first rows of that slice of Q (8 rows of bytes; of Y 4 rows of halves without Q), which the last
// launch reads before it writes them.  us, one launch / three, from HBM (600 MB of buffers in turn), residual and int8 output: 4096 rows, 32
// tokens 9.7 / 11.0, 64 tokens 14.4 / 11.5, 512 tokens 26 / 13.9 (from the last-level cache 18.0 / 12.8), 8192 tokens 81 / 66; 2500 rows, 64
// tokens 10.5 / 11.2, 1024 tokens 18.2 / 14.5; 8192 rows, 16 tokens 11.5 / 12.6, 256 tokens 42 / 15.2; 16384 rows, 8 tokens 68 / 16;
// 2048 rows, 1024 tokens 14.1 / 13.6 (11.2 / 12.5), 8192 tokens 40.7 / 37.5; 1024 rows, 8192 tokens 20.2 / 23.9, 16384 tokens 37.5 / 36.3.
// Without a residual: 4096 rows, 8192 tokens 40.9 / 43.1, with both outputs 63 / 55; 6000 rows, 64 tokens 11.1 / 11.9, 8192 tokens 60.3 /
// 59.7; 8192 rows, 64 tokens 14.1 / 12.3, 8192 tokens 86 / 76.  (Of 8 rows a lane in workgroups of 256 threads 72 where 2 rows in
// 1024 threads take 65.6.)
constexpr int SL_TOK = 128, SL_NT = 1024, SL_RPP = SL_NT / (SL_TOK / 8), SL_CH = 2;      // 64 rows at a time, twice
constexpr int SL_ROWS = SL_CH * SL_RPP;

static bool slices_fit(const NormArgs& g) {              // threads of a grid
  return (((int64_t)g.M + SL_TOK - 1) / SL_TOK) * ((g.K + SL_ROWS - 1) / SL_ROWS) * SL_NT <= 0xffffffffll;
}
static bool slices_pay(const NormArgs& g) {
  const int64_t values = (int64_t)g.M * g.K;
  if (!slices_fit(g)) return false;
  if (g.K > 8192) return true;
  if (g.R) return g.K > 2048 ? values >= 160000 : g.K >= 1024 && values >= 1 << 24;
  return g.K > 4096 ? values >= 400000 : g.K > 2048 && g.Y && g.Q && values >= 1 << 24;
}

__device__ __forceinline__ int slice_row(const NormArgs& g, int s, int n) { return (int)((int64_t)g.K * s / n); }

__device__ __forceinline__ uint2 get_sums(const NormArgs& g, int k, int m) {
  uint32_t w[2] = {0u, 0u};
  if (g.Q) {
    uint32_t b[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) b[j] = ((const uint8_t*)g.Q)[(size_t)(k + j) * g.ldq + m];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j >> 2] |= b[j] << (8 * (j & 3));
  } else {
    uint32_t b[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) b[j] = ((const uint16_t*)g.Y)[(size_t)(k + j) * g.ld + m];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j >> 1] |= b[j] << (16 * (j & 1));
  }
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void put_sums(const NormArgs& g, int k, int m, uint2 v) {
  if (g.Q) {
#pragma unroll
    for (int j = 0; j < 8; ++j) ((uint8_t*)g.Q)[(size_t)(k + j) * g.ldq + m] = (uint8_t)((j < 4 ? v.x : v.y) >> (8 * (j & 3)));
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) ((uint16_t*)g.Y)[(size_t)(k + j) * g.ld + m] = (uint16_t)((j < 2 ? v.x : v.y) >> (16 * (j & 1)));
  }
}

// What both kernels over slices know of their place.
struct SliceLane {
  int s, k0, k1, m0, m, c, r0, tail;
  bool live, whole;
  size_t at;
  __device__ __forceinline__ SliceLane(const NormArgs& g, int n) {
    const int bands = (g.M + SL_TOK - 1) / SL_TOK;
    s = (int)blockIdx.x / bands;
    m0 = ((int)blockIdx.x - s * bands) * SL_TOK;
    k0 = slice_row(g, s, n);
    k1 = slice_row(g, s + 1, n);
    c = threadIdx.x % (SL_TOK / 8);
    r0 = threadIdx.x / (SL_TOK / 8);
    m = m0 + c * 8;
    live = m < g.M;
    whole = m + 8 <= g.M;
    tail = g.M & 7;
    at = (size_t)(live ? m : m0);
  }
  __device__ __forceinline__ int row(int i) const { return k0 + r0 + i * SL_RPP; }
  __device__ __forceinline__ half8 load(const _Float16* from, const NormArgs& g, int i) const {
    return *(const half8*)(from + (size_t)min(row(i), k1 - 1) * g.ld + at);
  }
};

__global__ __launch_bounds__(SL_NT) void norm_slices_kernel(NormArgs g, int n) {
  constexpr int NW = SL_NT / 64;
  __shared__ float s_sum[NW][SL_TOK], s_top[NW][SL_TOK];
  const SliceLane a(g, n);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  half8 h[SL_CH];
  _Float16 gam[SL_CH];
#pragma unroll
  for (int i = 0; i < SL_CH; ++i) h[i] = a.load(g.X, g, i);
#pragma unroll
  for (int i = 0; i < SL_CH; ++i) gam[i] = (_Float16)1.f;
  if (g.gamma) {
#pragma unroll
    for (int i = 0; i < SL_CH; ++i) gam[i] = g.gamma[min(a.row(i), a.k1 - 1)];
  }
  if (g.R) {
    half8 r[SL_CH];
#pragma unroll
    for (int i = 0; i < SL_CH; ++i) r[i] = a.load(g.R, g, i);
#pragma unroll
    for (int i = 0; i < SL_CH; ++i) h[i] += r[i];
  }
  if (g.H) {
#pragma unroll
    for (int i = 0; i < SL_CH; ++i)
      if (a.row(i) < a.k1 && a.live) store8(g.H + (size_t)a.row(i) * g.ld + a.m, h[i], a.whole, a.tail);
  }
  float sum[8], top[8], worst = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) { sum[e] = 0.f; top[e] = 0.f; }
#pragma unroll
  for (int i = 0; i < SL_CH; ++i) {
    if (a.row(i) >= a.k1) h[i] = half8{0, 0, 0, 0, 0, 0, 0, 0};
    const float gm = (float)gam[i];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float f = (float)h[i][e];
      sum[e] = __builtin_fmaf(f, f, sum[e]);
      top[e] = __builtin_fmaxf(top[e], __builtin_fabsf(f * gm));
    }
    worst = __builtin_fmaf(gm, 0.f, worst);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) top[e] = worst == 0.f ? top[e] : __builtin_inff();      // (a gamma that is not finite: every token)
  halve(sum, [](float x, float y) { return x + y; });
  halve(top, [](float x, float y) { return __builtin_fmaxf(x, y); });
  const int tok = a.c * 8 + 2 * (lane >> 4 & 1) + 4 * (lane >> 5);
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    s_sum[wave][tok + e] = sum[e];
    s_top[wave][tok + e] = top[e];
  }
  __syncthreads();
  if (tid < SL_TOK && a.m0 + tid < g.M) {
    float x = s_sum[0][tid], t = s_top[0][tid];
#pragma unroll
    for (int w = 1; w < NW; ++w) {
      x += s_sum[w][tid];
      t = __builtin_fmaxf(t, s_top[w][tid]);
    }
    put_sums(g, a.k0, a.m0 + tid, make_uint2(__float_as_uint(x), x < __builtin_inff() ? __float_as_uint(t) : INF_BITS));
  }
}

// TK_TOK tokens, 16 groups of threads on the slices by turns: up to 32 slices (4096 rows) in one round trip.
constexpr int TK_GRP = 16;
template <bool NORM, int TK_TOK>
__global__ __launch_bounds__(TK_TOK * TK_GRP) void norm_tokens_kernel(NormArgs g, int n) {
  __shared__ float s_sum[TK_GRP][TK_TOK];
  __shared__ uint32_t s_top[TK_GRP][TK_TOK];
  __shared__ uint2 s_out[TK_TOK];
  const int tok = threadIdx.x % TK_TOK, grp = threadIdx.x / TK_TOK, m = (int)blockIdx.x * TK_TOK + tok;
  float sum = 0.f;
  uint32_t top = 0;
  if (m < g.M)
    for (int s = grp; s < n; s += 2 * TK_GRP) {
      const uint2 v = get_sums(g, slice_row(g, s, n), m);
      const uint2 w = get_sums(g, slice_row(g, min(s + TK_GRP, n - 1), n), m);
      sum += __uint_as_float(v.x);
      top = max(top, v.y);
      if (s + TK_GRP < n) {
        sum += __uint_as_float(w.x);
        top = max(top, w.y);
      }
    }
  s_sum[grp][tok] = sum;
  s_top[grp][tok] = top;
  __syncthreads();
  if (grp == 0) {
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < TK_GRP; ++w) {
      sum += s_sum[w][tok];
      top = max(top, s_top[w][tok]);
    }
    const Token t = finish_token<NORM>(sum, top, g);
    if (g.scale && m < g.M) g.scale[m] = t.scale;
    s_out[tok] = make_uint2(__float_as_uint(t.inv), top);
  }
  __syncthreads();
  if (m < g.M)
    for (int s = grp; s < n; s += TK_GRP) put_sums(g, slice_row(g, s, n), m, s_out[tok]);
}

__global__ __launch_bounds__(SL_NT) void norm_outputs_kernel(NormArgs g, int n) {
  __shared__ __attribute__((aligned(16))) float s_inv[SL_TOK], s_mul[SL_TOK], s_max[SL_TOK];
  const SliceLane a(g, n);
  const int tid = threadIdx.x;
  half8 h[SL_CH];
  _Float16 gam[SL_CH];
  const _Float16* from = g.H ? g.H : g.X;
#pragma unroll
  for (int i = 0; i < SL_CH; ++i) h[i] = a.load(from, g, i);
#pragma unroll
  for (int i = 0; i < SL_CH; ++i) gam[i] = (_Float16)1.f;
  if (g.gamma) {
#pragma unroll
    for (int i = 0; i < SL_CH; ++i) gam[i] = g.gamma[min(a.row(i), a.k1 - 1)];
  }
  if (g.R && !g.H) {
    half8 r[SL_CH];
#pragma unroll
    for (int i = 0; i < SL_CH; ++i) r[i] = a.load(g.R, g, i);
#pragma unroll
    for (int i = 0; i < SL_CH; ++i) h[i] += r[i];
  }
  if (tid < SL_TOK) {
    const uint2 v = a.m0 + tid < g.M ? get_sums(g, a.k0, a.m0 + tid) : make_uint2(0u, 0u);
    const float big = __uint_as_float(v.y);
    s_inv[tid] = __uint_as_float(v.x);
    s_max[tid] = big;
    s_mul[tid] = v.y != 0 && v.y < INF_BITS ? 127.f / big : 0.f;
  }
  __syncthreads();                       // every sum of the slice has been read; its rows are written now
  float inv[8], mul[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) { inv[e] = s_inv[a.c * 8 + e]; mul[e] = s_mul[a.c * 8 + e]; }
  if (!a.live) return;
  if (g.Y) {
#pragma unroll
    for (int i = 0; i < SL_CH; ++i) {
      half8 y;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = (_Float16)((float)h[i][e] * (float)gam[i] * inv[e]);
      if (a.row(i) < a.k1) store8(g.Y + (size_t)a.row(i) * g.ld + a.m, y, a.whole, a.tail);
    }
  }
  if (g.Q) {
#pragma unroll
    for (int i = 0; i < SL_CH; ++i) {
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = (float)h[i][e] * (float)gam[i];
      const uint2 q = round8(f, mul, s_max + a.c * 8);
      if (a.row(i) < a.k1) store8(g.Q + (size_t)a.row(i) * g.ldq + a.m, q, a.whole, a.tail);
    }
  }
}

// n slices of at most SL_ROWS and at least 8 rows.  (The quantiser is the norm's first and last launch without R and gamma.)
template <bool NORM>
hipError_t run_norm_slices(const NormArgs& g, int n, hipStream_t stream) {
  const unsigned bands = (unsigned)(((int64_t)g.M + SL_TOK - 1) / SL_TOK);
  hipError_t e = launch_kernel(norm_slices_kernel, dim3(bands * n), dim3(SL_NT), stream, g, n);
  // (64 tokens: 8192 x 4096 66.9 -> 65.6 us; 8192 x 128 13.9 -> 14.5)
  if (e == hipSuccess)
    e = g.M > 2048 ? launch_kernel(norm_tokens_kernel<NORM, 64>, dim3((unsigned)(((int64_t)g.M + 63) / 64)), dim3(64 * TK_GRP), stream, g, n)
                   : launch_kernel(norm_tokens_kernel<NORM, 32>, dim3((unsigned)((g.M + 31) / 32)), dim3(32 * TK_GRP), stream, g, n);
  if (e == hipSuccess) e = launch_kernel(norm_outputs_kernel, dim3(bands * n), dim3(SL_NT), stream, g, n);
  return e;
}

// Tokens per workgroup: 8 while that is at most one workgroup per CU (few rows of a token per lane and every CU at
// work), 16 up to two, then 32, whose pieces of a row are half a line of memory; where a workgroup fills a CU (above 2048
// rows) 32 for one round, whole lines for one round, then slices (not up to 2560 rows where the last round is well filled).  Rows in registers as far as they fit, fewer lanes where they would have
// nothing to do.  us with 8 / 16 / 32 / 64 tokens, int8 output, from HBM (600 MB of buffers in turn), with a residual: 768 rows, 2048 tokens
// 7.7 / 9.8 / 11.9 / 19, 4096 tokens 13.3 / 11.4 / 13.5 / 20, 6000 tokens 19.7 / 17.3 / 14.8 / 23; 1024 rows, 8192 tokens 29 / 24 / 20 / 27; 2048
// rows, 2500 tokens 26 / 20 / 26 / 41; 4096 rows, 16 tokens 7.1 / 9.5 / 20 / 36 (buffers that the last-level cache holds: 768 rows, 4096
// tokens 10.8 / 8.2 / 9.5).  Without: 4096 rows, 1024 tokens 13.4 / 17.9 / 27 / 39, 4096 tokens 29 / 23 / 33 / 44, 8192 tokens 50 / 45 / 41 / 47,
// 9000 tokens 66 / 57 / 72 / 57 (slices 56), 16000 tokens 97 / 75 / 72 / 72 (75), 17000 tokens 120 / 96 / 115 / 124 (95); 2100 rows, 9000
// tokens 35 / 33 / 43 / 34 (35), 16000 tokens 52 / 46 / 43 / 34 (45), 18000 tokens 63 / 57 / 71 / 72 (58), 24000 tokens 73 / 64 / 63 / 60 (62).
template <bool NORM>
static hipError_t dispatch_norm(const NormArgs& g, hipStream_t stream) {
  const int K = g.K;
  if (slices_pay(g)) return run_norm_slices<NORM>(g, (K + SL_ROWS - 1) / SL_ROWS, stream);
  if (g.M <= 2048 && K <= 8192) {
    if (K <= 1024) return run_norm<NORM, 8, 512, 2>(g, stream);
    if (K <= 2048) return run_norm<NORM, 8, 512, 4>(g, stream);
    if (K <= 4096) return run_norm<NORM, 8, 1024, 4>(g, stream);
    return run_norm<NORM, 8, 1024, 8>(g, stream);
  }
  if (g.M <= 4096 && K <= 4096) {
    if (K <= 1024) return run_norm<NORM, 16, 1024, 2>(g, stream);
    if (K <= 2048) return run_norm<NORM, 16, 1024, 4>(g, stream);
    return run_norm<NORM, 16, 1024, 8>(g, stream);
  }
  if (g.M < 1 << 25) {                   // (2^32 threads in a grid: none of 32 tokens beyond 2^27 - 1)
    if (K <= 1024) return run_norm<NORM, 32, 1024, 4>(g, stream);
    if (K <= 2048) return run_norm<NORM, 32, 1024, 8>(g, stream);
    // Half of the rows in LDS: the quantiser, 8192 tokens x 4096, 35 us against 41 read again and 41 in slices (a copy 18.3: all
    // of a workgroup's loads come before its stores, and its 128 KiB of LDS leave a CU no second one; the stores are pieces of
    // 32 bytes); 17000 tokens 87, 108, 92.  The norm spills registers there.
    if (!NORM && K <= 4096) return run_norm<NORM, 32, 1024, 8, 8>(g, stream);
    if constexpr (NORM)
      if (g.M <= 8192) return run_norm<NORM, 32, 1024, 0>(g, stream);
  }
  if (K > 2048 && g.M > 16384 && (K > 2560 || g.M % 16384 < 6144) && slices_fit(g))
    return run_norm_slices<NORM>(g, (K + SL_ROWS - 1) / SL_ROWS, stream);
  return run_norm<NORM, 64, 1024, 0>(g, stream);
}

hipError_t launch_norm(bool norm, const NormArgs& g, hipStream_t stream) {
  return norm ? dispatch_norm<true>(g, stream) : dispatch_norm<false>(g, stream);
}

}  // namespace twg
