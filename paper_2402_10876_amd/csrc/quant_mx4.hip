// Quantiser of activations to microscaled 4-bit floating point (format in mx4_format.h).
//
// Per token and 32 rows: the largest magnitude gives the power of two (an integer maximum over the fp16 bits, which order as
// the magnitudes do, infinities and NaN on top), v_cvt_scalef32_pk_fp4_f16 rounds two values at a time (nearest even,
// past 6 to 6; checked for every fp16 value against the definition).  Bound by memory: 2 bytes in and 17/32 out per value.
//   K x M : a lane takes two neighbouring tokens, 32 loads of 4 bytes, all under way at once; a wave reads 256 bytes of
//           each row and writes 2 KiB of codes in a run.  With few values a lane takes 4 rows, so that there are lanes at work and
//           no lane has 32 loads to issue.
//   M x K : a wave takes 16 blocks of 4 tokens, 1 KiB of a token per load; four lanes hold a block, whose codes are
//           collected in LDS so that the writes are runs of 64 bytes (4 tokens of a block row).  Workgroups that start
//           together read whole tokens: side by side down the rows they meet the same channels of memory where a row
//           is a power of two of bytes.  us, tokens first / whole tokens: 8192 x 4096 20.0 / 17.2 (a copy 15.4), 8192 x 2048 12.2 / 10.5 (7.7;
//           from the last-level cache 10.2 / 7.9), 8192 x 1024 6.5 / 6.5, 4096 x 768 4.5 / 4.4; waves of 8 tokens 8192 x 4096 20.9 / 18.0.
#include <type_traits>

#include "device_common.h"
#include "fewbit.h"
#include "grid.h"
#include "mx4_format.h"

namespace twg {

namespace {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));

// Scale byte of a block whose largest magnitude has the fp16 bits `top`.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  if (top >= 0x7c00u) return MX4_NAN;
  if (top == 0) return MX4_ONE;
  const float f = (float)__builtin_bit_cast(_Float16, (unsigned short)top);
  return (__float_as_uint(f) >> 23) - 2;
}

// 4 pairs of fp16 values (rows 2i, 2i+1) to 8 codes.
__device__ __forceinline__ uint32_t encode8(const uint32_t (&x)[4], float scale) {
  uint32_t o = 0;
  o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(o, __builtin_bit_cast(half2v, x[0]), scale, 0);
  o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(o, __builtin_bit_cast(half2v, x[1]), scale, 1);
  o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(o, __builtin_bit_cast(half2v, x[2]), scale, 2);
  o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(o, __builtin_bit_cast(half2v, x[3]), scale, 3);
  return o;
}

// 16 pairs of fp16 values (rows 2i, 2i+1) to 32 codes; a block that is not finite gets zeros.
__device__ __forceinline__ u32x4 encode(const uint32_t (&x)[16], uint32_t scale) {
  const float s = __uint_as_float((scale == MX4_NAN ? MX4_ONE : scale) << 23);
  u32x4 out;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w[4] = {x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
    out[i] = scale == MX4_NAN ? 0u : encode8(w, s);
  }
  return out;
}

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  const ushort2v x = __builtin_bit_cast(ushort2v, a), y = __builtin_bit_cast(ushort2v, b);
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(x, y));
}

}  // namespace

// K x M.  One wave: 128 tokens x one block of rows; neighbouring workgroups along the rows (n_rows of them) or along the tokens.
// us along rows / tokens, from HBM: 4096 x 768 4.3 / 4.2, 5000 x 1003 5.35 / 5.8, 8192 x 1024 6.5 / 6.4, 8192 x 4096 20.7 / 19.8.
__global__ __launch_bounds__(256) void quant_mx4_km_kernel(QuantMx4Args g, int n_blocks, int n_rows, int n_tokens) {
  const int lane = threadIdx.x & 63;
  const int bid = (int)(blockIdx.y * gridDim.x + blockIdx.x);      // (those past the last one: no block or no token)
  const int at_rows = n_rows ? bid % n_rows : bid / n_tokens, at_tokens = n_rows ? bid / n_rows : bid % n_tokens;
  const int b = at_rows * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m = (at_tokens * 64 + lane) * 2;
  if (b >= n_blocks || m >= g.M) return;
  const int k0 = b * MX4_BLOCK, rows = min(g.K - k0, MX4_BLOCK);
  const _Float16* x = g.X + (size_t)k0 * g.ldx + m;
  uint32_t v[32];
#pragma unroll
  for (int k = 0; k < 32; ++k) {        // (rows behind K: the last one again, then zeros)
    v[k] = *(const uint32_t*)(x + (size_t)min(k, rows - 1) * g.ldx);
    if (k >= rows) v[k] = 0;
  }
  uint32_t top = 0;
#pragma unroll
  for (int k = 0; k < 32; ++k) top = max_u16x2(top, v[k] & 0x7fff7fffu);
  uint32_t lo[16], hi[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    lo[i] = __builtin_amdgcn_perm(v[2 * i + 1], v[2 * i], 0x05040100u);
    hi[i] = __builtin_amdgcn_perm(v[2 * i + 1], v[2 * i], 0x07060302u);
  }
  const uint32_t s0 = scale_byte(top & 0xffffu), s1 = scale_byte(top >> 16);
  const size_t at = (size_t)b * g.ldq + m;
  *(u32x4*)(g.Q + at * 16) = encode(lo, s0);
  if (m + 1 < g.M) {
    *(u32x4*)(g.Q + at * 16 + 16) = encode(hi, s1);
    *(uint16_t*)(g.S + at) = (uint16_t)(s0 | s1 << 8);
  } else {
    g.S[at] = (uint8_t)s0;
  }
}

// K x M, few values.  One wave: 16 tokens x one block of rows; a lane takes two tokens and 4 rows.  us, 32 rows a lane / 4 rows: 1 x
// 4096 3.4 / 1.9, 16 x 4096 3.9 / 2.0, 128 x 1024 2.6 / 2.0, 1024 x 1024 3.15 / 2.75, 1957 x 1003 3.8 / 3.5, 2048 x 1024 3.75 / 4.1, 4096 x 768
// 4.25 / 6.5.
__global__ __launch_bounds__(256) void quant_mx4_few_kernel(QuantMx4Args g, int n_blocks, int n_rows) {
  const int lane = threadIdx.x & 63, pair = lane & 7, part = lane >> 3;
  const int at_tokens = (int)blockIdx.x / n_rows, at_rows = (int)blockIdx.x - at_tokens * n_rows;
  const int b = at_rows * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m = at_tokens * 16 + pair * 2, k = b * MX4_BLOCK + part * 4;
  if (b >= n_blocks) return;
  const _Float16* x = g.X + (m < g.M ? m : 0);
  uint32_t v[4], top = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = *(const uint32_t*)(x + (size_t)min(k + j, g.K - 1) * g.ldx);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (k + j >= g.K) v[j] = 0;
    top = max_u16x2(top, v[j] & 0x7fff7fffu);
  }
  top = max_u16x2(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x128, 0xf, 0xf, true));      // row_ror:8
  const auto t16 = __builtin_amdgcn_permlane16_swap(top, top, false, false);
  top = max_u16x2(t16[0], t16[1]);
  const auto t32 = __builtin_amdgcn_permlane32_swap(top, top, false, false);
  top = max_u16x2(t32[0], t32[1]);
  if (m >= g.M) return;
  const size_t at = (size_t)b * g.ldq + m;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    if (m + t >= g.M) break;
    const uint32_t sel = t ? 0x07060302u : 0x05040100u, s = scale_byte(t ? top >> 16 : top & 0xffffu);
    const float f = __uint_as_float((s == MX4_NAN ? MX4_ONE : s) << 23);
    const uint32_t lo = __builtin_amdgcn_perm(v[1], v[0], sel), hi = __builtin_amdgcn_perm(v[3], v[2], sel);
    uint32_t o = 0;
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(o, __builtin_bit_cast(half2v, lo), f, 0);
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(o, __builtin_bit_cast(half2v, hi), f, 1);
    *(uint16_t*)(g.Q + (at + t) * 16 + part * 2) = s == MX4_NAN ? 0 : (uint16_t)o;
    if (part == 0) g.S[at + t] = (uint8_t)s;
  }
}

// M x K.  One wave: TOK tokens x 16 blocks; four lanes hold a block of a token.
constexpr int TOK = 4;
__global__ __launch_bounds__(256) void quant_mx4_mk_kernel(QuantMx4Args g, int n_blocks, uint32_t n_cols) {
  __shared__ __attribute__((aligned(16))) uint32_t codes[4][16 * TOK * 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t bid = blockIdx.y * gridDim.x + blockIdx.x;        // (those past the last one: m0 >= M)
  const int at_tokens = (int)(bid / n_cols), at_cols = (int)(bid % n_cols);
  const int m0 = (at_tokens * 4 + wave) * TOK, b0 = at_cols * 16;
  if (m0 >= g.M) return;
  const int k = b0 * MX4_BLOCK + lane * 8, left = g.K - k;         // values of the lane in front of K: left and more
  const _Float16* x = g.X + (size_t)m0 * g.ldx + (left > 0 ? k : 0);
  u32x4 v[TOK];
#pragma unroll
  for (int t = 0; t < TOK; ++t) v[t] = *(const u32x4*)(x + (size_t)min(t, g.M - 1 - m0) * g.ldx);
  if (left < 8) {
#pragma unroll
    for (int t = 0; t < TOK; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) v[t][j] = 2 * j + 1 < left ? v[t][j] : 2 * j < left ? v[t][j] & 0xffffu : 0u;
  }
  uint32_t scales[TOK / 4] = {};
#pragma unroll
  for (int t = 0; t < TOK; ++t) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) top = max_u16x2(top, v[t][j] & 0x7fff7fffu);
    top = max(top & 0xffffu, top >> 16);
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xb1, 0xf, 0xf, true));     // quad_perm [1,0,3,2]
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4e, 0xf, 0xf, true));     // quad_perm [2,3,0,1]
    const uint32_t s = scale_byte(top);
    scales[t / 4] |= s << (8 * (t % 4));
    const float f = __uint_as_float((s == MX4_NAN ? MX4_ONE : s) << 23);
    const uint32_t w[4] = {v[t][0], v[t][1], v[t][2], v[t][3]};      // (a bit cast of a vector's element takes the first one)
    const uint32_t o = encode8(w, f);
    codes[wave][((lane >> 2) * TOK + t) * 4 + (lane & 3)] = s == MX4_NAN ? 0u : o;
  }
  // (an area of the wave's own: LDS instructions of a wave are done in order)
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int i = 0; i < TOK / 4; ++i) {
    const int p = i * 64 + lane, b = b0 + p / TOK, m = m0 + p % TOK;
    const u32x4 c = *(const u32x4*)&codes[wave][p * 4];
    if (b < n_blocks && m < g.M) *(u32x4*)(g.Q + ((size_t)b * g.ldq + m) * 16) = c;
  }
  const int b = b0 + (lane >> 2);
  if ((lane & 3) == 0 && b < n_blocks) {
    uint8_t* to = g.S + (size_t)b * g.ldq + m0;
#pragma unroll
    for (int i = 0; i < TOK / 4; ++i) {
      if (m0 + 4 * i + 4 <= g.M) *(uint32_t*)(to + 4 * i) = scales[i];
      else
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (m0 + 4 * i + e < g.M) to[4 * i + e] = (uint8_t)(scales[i] >> (8 * e));
    }
  }
}

hipError_t launch_quant_mx4(bool km, const QuantMx4Args& g, hipStream_t stream) {
  const int nb = (g.K + MX4_BLOCK - 1) / MX4_BLOCK;
  const int64_t values = (int64_t)g.M * g.K;
  const bool few = km && values < 1 << 21;
  const int64_t per = few ? 16 : km ? 128 : 4 * TOK;
  const int64_t n_tokens = (g.M + per - 1) / per, n_other = km ? (nb + 3) / 4 : (nb + 15) / 16;
  // (2^27 row-major tokens of more than 512 values are more threads than one dimension takes)
  const Grid2 n = grid_of((uint64_t)(n_tokens * n_other), 256);
  const dim3 grid(n.x, n.y);
  if (few) return launch_kernel(quant_mx4_few_kernel, grid, dim3(256), stream, g, nb, (int)n_other);
  if (km) return launch_kernel(quant_mx4_km_kernel, grid, dim3(256), stream, g, nb, values < 8 << 20 ? (int)n_other : 0, (int)n_tokens);
  return launch_kernel(quant_mx4_mk_kernel, grid, dim3(256), stream, g, nb, (uint32_t)n_other);
}

}  // namespace twg
