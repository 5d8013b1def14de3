// Root-mean-square norm with the residual's addition, output in int8 with a scale per token and / or in fp16, and the int8
// quantiser alone.  K x M activations: a token is a column, its K values ld elements apart.
//
//   h = fp16(x + r);  g = h * gamma (exact in fp32: two 11-bit mantissas);  inv = 1 / sqrt(mean h^2 + eps)
//   y = fp16(g * inv);  scale = max |g| * inv / 127;  q = nearest integer of 127 g / max |g|, ties to even
//
// inv cancels in q, which is therefore exact: u = fma(g, fl(127 / max|g|), 1.5 * 2^23) rounds to an integer in the low byte of
// u, wrong only within 127 * 2^-24 of a half; where the distance to n is more than 0.4999 the side is settled in 64 bits
// (254 g against (2n +- 1) max|g|, both exact).  Sums of squares are fp32 (at most 32 terms a lane, then a tree).
//
// Bound by memory: 2 bytes in per value (4 with a residual), 1 to 5 out.  One workgroup owns 32 tokens and all K rows and
// keeps its values in registers between the two passes, up to 16 rows a lane; longer columns are read again, from L2.
#include <type_traits>

#include "device_common.h"
#include "fewbit.h"

namespace twg {

namespace {

constexpr int TOK = 32;                  // tokens of a workgroup: 64 bytes of every row
constexpr int LPR = TOK / 8;             // lanes per row, 8 tokens each
constexpr float MAGIC = 12582912.f;      // 1.5 * 2^23

// The integer nearest to 127 g / top where n is next to a half away (d: which side).
__device__ __forceinline__ float settle(float g, float top, float n, float d) {
  const double sgn = d > 0.f ? 1.0 : -1.0;
  const double x = 254.0 * (double)g, edge = (2.0 * (double)n + sgn) * (double)top;
  const bool odd = ((int)n & 1) != 0;
  if (d > 0.f) return (x > edge || (x == edge && odd)) ? n + 1.f : n;
  return (x < edge || (x == edge && odd)) ? n - 1.f : n;
}

}  // namespace

// NT threads; NCH: rows a lane keeps (0: more than fit, the second pass reads them again).
template <bool NORM, int NT, int NCH>
__global__ __launch_bounds__(NT) void norm_kernel(NormArgs g) {
  constexpr int RPP = NT / LPR;          // rows per pass
  constexpr int NW = NT / 64;
  __shared__ float s_sum[NW][TOK];
  __shared__ uint32_t s_top[NW][TOK];
  __shared__ float s_inv[TOK], s_mul[TOK], s_max[TOK];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int m0 = xcd_remap(blockIdx.x, gridDim.x) * TOK;
  const int c = tid % LPR, r0 = tid / LPR;
  const int m = m0 + c * 8;
  const bool live = m < g.M;
  const size_t at = live ? (size_t)m : (size_t)m0;
  const bool whole = m + 8 <= g.M;
  const int n_ch = (g.K + RPP - 1) / RPP;

  auto load_h = [&](int i) {             // rows behind K: zeros
    const int k = r0 + i * RPP, kc = min(k, g.K - 1);
    half8 x = *(const half8*)(g.X + (size_t)kc * g.ld + at);
    if (NORM && g.R) x += *(const half8*)(g.R + (size_t)kc * g.ld + at);
    if (k >= g.K) x = half8{0, 0, 0, 0, 0, 0, 0, 0};
    return x;
  };
  auto gamma_of = [&](int i) -> float {
    if constexpr (!NORM) return 1.f;
    return g.gamma ? (float)g.gamma[min(r0 + i * RPP, g.K - 1)] : 1.f;
  };
  auto store_half = [&](_Float16* to, int i, half8 v) {
    const int k = r0 + i * RPP;
    if (k >= g.K || !live) return;
    _Float16* p = to + (size_t)k * g.ld + m;
    if (whole) *(half8*)p = v;
    else
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (m + e < g.M) p[e] = v[e];
  };

  float sum[8];
  uint32_t top[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) { sum[e] = 0.f; top[e] = 0u; }
  auto stats = [&](half8 h, float gam) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float f = (float)h[e];
      if constexpr (NORM) sum[e] = __builtin_fmaf(f, f, sum[e]);
      top[e] = max(top[e], __float_as_uint(f * gam) & 0x7fffffffu);      // (NaN above infinity above the numbers)
    }
  };

  half8 keep[NCH ? NCH : 1];
  float gam[NCH ? NCH : 1];
  if constexpr (NCH > 0) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) { keep[i] = load_h(i); gam[i] = gamma_of(i); }
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      if (NORM && g.H) store_half(g.H, i, keep[i]);
      stats(keep[i], gam[i]);
    }
  } else {
    for (int i = 0; i < n_ch; ++i) {
      const half8 h = load_h(i);
      if (NORM && g.H) store_half(g.H, i, h);
      stats(h, gamma_of(i));
    }
  }

  // sums and maxima over the lanes with the same tokens, then over the waves
#pragma unroll
  for (int d = LPR; d < 64; d *= 2)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (NORM) sum[e] += __shfl_xor(sum[e], d);
      top[e] = max(top[e], (uint32_t)__shfl_xor((int)top[e], d));
    }
  if (lane < LPR)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (NORM) s_sum[wave][lane * 8 + e] = sum[e];
      s_top[wave][lane * 8 + e] = top[e];
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
    float inv = 1.f;
    if constexpr (NORM) inv = 1.f / sqrtf(s / (float)g.K + g.eps);
    const bool fine = t != 0 && t < 0x7f800000u;
    const float big = __uint_as_float(t);
    s_inv[tid] = inv;
    s_max[tid] = big;
    s_mul[tid] = fine ? 127.f / big : 0.f;
    if (g.scale && m0 + tid < g.M)
      g.scale[m0 + tid] = fine ? big * inv / 127.f : t == 0 ? 0.f : __builtin_nanf("");
  }
  __syncthreads();
  float inv[8], mul[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) { inv[e] = s_inv[c * 8 + e]; mul[e] = s_mul[c * 8 + e]; }

  auto finish = [&](int i, half8 h, float gm) {
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (float)h[e] * gm;
    if (NORM && g.Y) {
      half8 y;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = (_Float16)(f[e] * inv[e]);
      store_half(g.Y, i, y);
    }
    if (!g.Q) return;
    float u[8], d[8], far = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      u[e] = __builtin_fmaf(f[e], mul[e], MAGIC);
      d[e] = __builtin_fmaf(f[e], mul[e], -(u[e] - MAGIC));
      far = __builtin_fmaxf(far, __builtin_fabsf(d[e]));
    }
    if (far > 0.4999f) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (__builtin_fabsf(d[e]) > 0.4999f) u[e] = settle(f[e], s_max[c * 8 + e], u[e] - MAGIC, d[e]) + MAGIC;
    }
    uint32_t q[2] = {0u, 0u};
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e >> 2] |= (__float_as_uint(u[e]) & 0xffu) << (8 * (e & 3));
    const int k = r0 + i * RPP;
    if (k >= g.K || !live) return;
    int8_t* p = g.Q + (size_t)k * g.ldq + m;
    if (whole) *(uint2*)p = make_uint2(q[0], q[1]);
    else
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (m + e < g.M) p[e] = (int8_t)(q[e >> 2] >> (8 * (e & 3)));
  };
  if constexpr (NCH > 0) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) finish(i, keep[i], gam[i]);
  } else {
    for (int i = 0; i < n_ch; ++i) {
      half8 h;
      if (NORM && g.H) {                 // (this lane's own stores; X or R may be the same buffer)
        const int k = r0 + i * RPP, kc = min(k, g.K - 1);
        h = half8{0, 0, 0, 0, 0, 0, 0, 0};
        if (k < g.K && live) {
          const _Float16* p = g.H + (size_t)kc * g.ld + m;
          if (whole) h = *(const half8*)p;
          else
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (m + e < g.M) h[e] = p[e];
        }
      } else {
        h = load_h(i);
      }
      finish(i, h, gamma_of(i));
    }
  }
}

template <bool NORM>
static hipError_t dispatch_norm(const NormArgs& g, hipStream_t stream) {
  const dim3 grid((unsigned)(((int64_t)g.M + TOK - 1) / TOK));
  if (g.K <= 512) return launch_kernel(norm_kernel<NORM, 512, 4>, grid, dim3(512), stream, g);
  if (g.K <= 1024) return launch_kernel(norm_kernel<NORM, 512, 8>, grid, dim3(512), stream, g);
  if (g.K <= 2048) return launch_kernel(norm_kernel<NORM, 512, 16>, grid, dim3(512), stream, g);
  return launch_kernel(norm_kernel<NORM, 512, 0>, grid, dim3(512), stream, g);
}

hipError_t launch_norm(bool norm, const NormArgs& g, hipStream_t stream) {
  return norm ? dispatch_norm<true>(g, stream) : dispatch_norm<false>(g, stream);
}

}  // namespace twg
