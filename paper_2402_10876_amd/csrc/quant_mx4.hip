// Quantiser of activations to microscaled 4-bit floating point (format in mx4_format.h).
//
// Per token and 32 rows: the largest magnitude gives the power of two (an integer maximum over the fp16 bits, which order as
// the magnitudes do, infinities and NaN on top), v_cvt_scalef32_pk_fp4_f16 rounds two values at a time (nearest even,
// past 6 to 6; checked for every fp16 value against the definition).  Bound by memory: 2 bytes in and 17/32 out per value.
//   K x M : a lane takes two neighbouring tokens, 32 loads of 4 bytes, all under way at once; a wave reads 256 bytes of
//           each row and writes 2 KiB of codes in a run.
//   M x K : a lane takes one block of a token, 64 bytes in a run; a wave is 8 tokens x 8 blocks, so that both
//           the reads (512 bytes of a token) and the writes (128 bytes of a block row) are whole lines.
#include <type_traits>

#include "device_common.h"
#include "fewbit.h"
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

// 16 pairs of fp16 values (rows 2i, 2i+1) to 32 codes; a block that is not finite gets zeros.
__device__ __forceinline__ u32x4 encode(const uint32_t (&x)[16], uint32_t scale) {
  const float s = __uint_as_float((scale == MX4_NAN ? MX4_ONE : scale) << 23);
  u32x4 out;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t o = 0;
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(o, __builtin_bit_cast(half2v, x[4 * i]), s, 0);
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(o, __builtin_bit_cast(half2v, x[4 * i + 1]), s, 1);
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(o, __builtin_bit_cast(half2v, x[4 * i + 2]), s, 2);
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(o, __builtin_bit_cast(half2v, x[4 * i + 3]), s, 3);
    out[i] = scale == MX4_NAN ? 0u : o;
  }
  return out;
}

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  const ushort2v x = __builtin_bit_cast(ushort2v, a), y = __builtin_bit_cast(ushort2v, b);
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(x, y));
}

}  // namespace

// K x M.  One wave: 128 tokens x one block of rows.
__global__ __launch_bounds__(256) void quant_mx4_km_kernel(QuantMx4Args g, int n_blocks) {
  const int lane = threadIdx.x & 63;
  const int b = blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m = ((int)blockIdx.x * 64 + lane) * 2;
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

// M x K.  One wave: 8 tokens x 8 blocks.
__global__ __launch_bounds__(256) void quant_mx4_mk_kernel(QuantMx4Args g, int n_blocks) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m = ((int)blockIdx.x * 4 + wave) * 8 + (lane & 7), b = (int)blockIdx.y * 8 + (lane >> 3);
  if (m >= g.M || b >= n_blocks) return;
  const int k0 = b * MX4_BLOCK, rows = g.K - k0;
  const _Float16* x = g.X + (size_t)m * g.ldx + k0;
  uint32_t v[16];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    u32x4 w = {0u, 0u, 0u, 0u};
    if (8 * i < rows) w = *(const u32x4*)(x + 8 * i);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int k = 8 * i + 2 * j;
      v[4 * i + j] = k + 1 < rows ? w[j] : k < rows ? w[j] & 0xffffu : 0u;
    }
  }
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) top = max_u16x2(top, v[i] & 0x7fff7fffu);
  const uint32_t s = scale_byte(max(top & 0xffffu, top >> 16));
  const size_t at = (size_t)b * g.ldq + m;
  *(u32x4*)(g.Q + at * 16) = encode(v, s);
  g.S[at] = (uint8_t)s;
}

hipError_t launch_quant_mx4(bool km, const QuantMx4Args& g, hipStream_t stream) {
  const int nb = (g.K + MX4_BLOCK - 1) / MX4_BLOCK;
  if (km)
    return launch_kernel(quant_mx4_km_kernel, dim3((unsigned)(((int64_t)g.M + 127) / 128), (nb + 3) / 4), dim3(256), stream, g, nb);
  return launch_kernel(quant_mx4_mk_kernel, dim3((unsigned)(((int64_t)g.M + 31) / 32), (nb + 7) / 8), dim3(256), stream, g, nb);
}

}  // namespace twg
