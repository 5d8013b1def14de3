// Internal: argument blocks and launchers of the few-bit operators (host side sees only this).
#pragma once
#include <hip/hip_runtime_api.h>
#include <stdint.h>

#include "packed.h"

namespace twg {

// Norm and int8 quantiser (norm.hip): K x M fp16, element (m, k) at X[k*ld + m].
struct NormArgs {
  const _Float16 *X, *R;         // R: residual or null
  const _Float16* gamma;         // K or null (ones)
  _Float16 *H, *Y;               // residual sum, normalised output; either may be null
  int8_t* Q;                     // int8 values and their scales, or both null
  float* scale;
  int M, K, ld, ldq;
  float eps;
};
// norm = false: the quantiser alone (R, gamma, H and Y are null, eps is not read).
hipError_t launch_norm(bool norm, const NormArgs& g, hipStream_t stream);

// 4-bit quantiser (quant_mx4.hip): blocks of 32 rows; codes Q[(b*ldq + m)*16 ..], scale bytes S[b*ldq + m].
struct QuantMx4Args {
  const _Float16* X;             // km: X[k*ldx + m]; else X[m*ldx + k]
  uint8_t *Q, *S;
  int M, K, ldx, ldq;
};
hipError_t launch_quant_mx4(bool km, const QuantMx4Args& g, hipStream_t stream);

// 4-bit products (gemm_mx4.hip).
struct GemmMx4Args {
  const uint8_t *Q, *S;          // activations as the quantiser writes them
  _Float16* C;                   // N x M, element (m, n) at C[n*ldc + m]
  int M, ldq, ldc;
  const Mx4Tile* tiles;
  const uint16_t* blocks;
  const int32_t *col_idx, *zero_cols;
  const uint8_t *vals, *wscale;
  int list_len;                  // entries of `blocks` per tile
  int n_tiles;                   // grouped: of a member
  const int32_t* offsets;        // grouped: n_members + 1 first tokens, else null
  int n_members, member_n;       // grouped: columns of a member
};
hipError_t launch_gemm_mx4(int G, GemmMx4Args g, hipStream_t stream);

}  // namespace twg
