// Products of microscaled 4-bit activations and weights on v_mfma_scale_f32_32x32x64_f8f6f4 (both operands e2m1, a power of
// two per 32 values applied by the instruction): C = A . W over the blocks of 32 rows that a tile of G columns keeps.
//
// Lane l of the instruction holds row l % 32 of its operand and the 32 values of block l / 32, 16 bytes, with their scale in a
// byte of another register.  That is the activations' layout in memory, 16 bytes per token and block with the tokens of
// a block row in a run, and the packer writes the weights the same way: both operands go from memory to registers with
// no LDS in between, a skipped block is a run that is not read, and tokens may start anywhere (a range of an expert).
// The list of kept blocks lies in LDS, so that addresses never wait for a load that is queued behind the operands'.
//
// A workgroup owns 32 MB WM tokens x 32 NB WN columns; WK waves deal the steps (two blocks) of a tile among themselves and
// add up in LDS.  Sums are fp32, one rounding to fp16.  The tile of C is turned round in LDS: 16-byte stores along the tokens.
#include <type_traits>

#include "device_common.h"
#include "fewbit.h"

namespace twg {

namespace {

typedef int int4v __attribute__((ext_vector_type(4)));
typedef int int8v __attribute__((ext_vector_type(8)));

constexpr int MAX_BLOCKS = 4096;         // of a column: K <= 131072

__device__ __forceinline__ int8v widen(int4v x) {
  return int8v{x[0], x[1], x[2], x[3], 0, 0, 0, 0};
}

template <int J>
__device__ __forceinline__ floatx16 mfma4(int4v a, int4v b, floatx16 c, int sa, int sb) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(widen(a), widen(b), c, 4, 4, 0, sa, J, sb);
}

// The tokens of M-tile mt when they are shared out by expert: expert e owns [offsets[e], offsets[e+1]) (cut to [0, M); an
// end in front of its start: none) in tiles of TM that start on a multiple of 8.  Every wave finds it by itself.
struct Range { int e, m0, lo, hi; };
__device__ __forceinline__ bool find_range(const GemmMx4Args& g, int mt, int TM, int lane, Range& r) {
  int before = 0;
  for (int c = 0; c < g.n_members; c += 64) {
    const int e = c + lane;
    int a = 0, b = 0;
    if (e < g.n_members) {
      a = min(max(g.offsets[e], 0), g.M);
      b = min(max(g.offsets[e + 1], 0), g.M);
    }
    const int tiles = b > a ? (b - (a & ~7) + TM - 1) / TM : 0;
    int incl = tiles;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int x = __shfl_up(incl, d);
      if (lane >= d) incl += x;
    }
    const unsigned long long hit = __ballot(before + incl > mt);
    if (hit) {
      const int f = __ffsll((long long)hit) - 1;
      const int start = before + __builtin_amdgcn_readlane(incl - tiles, f);
      const int af = __builtin_amdgcn_readlane(a, f);
      r.e = c + f;
      r.m0 = (af & ~7) + (mt - start) * TM;
      r.lo = max(af, r.m0);
      r.hi = __builtin_amdgcn_readlane(b, f);
      return true;
    }
    before += __builtin_amdgcn_readlane(incl, 63);
  }
  return false;
}

}  // namespace

template <int GB, int MB, int NB, int WM, int WN, int WK, int D>
__global__ __launch_bounds__(64 * WM * WN * WK, (MB * NB >= 8 ? 2 : 1)) void gemm_mx4_kernel(GemmMx4Args g) {
  constexpr int NT = 64 * WM * WN * WK;
  constexpr int TM = 32 * MB * WM, CB = NB * WN;            // tokens, column blocks of the workgroup
  constexpr int SUB = GB / CB;                              // workgroups per tile of columns
  static_assert(GB % CB == 0 && (WK == 1 || (MB == 1 && NB == 1)), "");
  // staged output: WK = 1 a wave's halves [n][m], else the waves' fp32 partial sums [wave][n][m]
  constexpr int PITCH = WK == 1 ? 32 * MB * 2 + 16 : 36 * 4;
  constexpr int AREA = 32 * NB * PITCH;
  __shared__ __attribute__((aligned(16))) char stage[WM * WN * WK * AREA];
  __shared__ uint16_t list[MAX_BLOCKS];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % WM, wn = wave / WM % WN, wk = wave / (WM * WN);
  const int nt = g.n_tiles * SUB;
  const int lid = xcd_remap(blockIdx.x, gridDim.x);
  const int mt = lid / nt;
  int t = (lid - mt * nt) / SUB;
  const int sub = (lid - mt * nt) % SUB;

  Range r{0, mt * TM, mt * TM, g.M};
  int col_base = 0;
  if (g.offsets) {
    if (!find_range(g, mt, TM, lane, r)) return;
    col_base = g.member_col[r.e];
    t += g.member_tile[r.e];
    if (t >= g.member_tile[r.e + 1]) return;
  }
  const int m0 = r.m0, m_end = min(r.hi, m0 + TM);
  const Mx4Tile tile = g.tiles[t];
  const int ns = tile.steps;
  for (int i = tid; i < 2 * ns; i += NT) list[i] = g.blocks[2 * tile.step0 + i];

  // pruned columns: 0
  {
    const int p0 = (r.lo - m0) >> 3, np = ((m_end - m0 + 7) >> 3) - p0;
    const int nz = tile.zero_end - tile.zero_beg;
    const int z0 = tile.zero_beg + (int)((int64_t)nz * sub / SUB), z1 = tile.zero_beg + (int)((int64_t)nz * (sub + 1) / SUB);
    for (int i = tid; i < (z1 - z0) * np; i += NT) {
      const int z = i / np, m = m0 + (p0 + i - z * np) * 8;
      _Float16* to = g.C + (size_t)(g.zero_cols[z0 + z] - col_base) * g.ldc + m;
      if (m >= r.lo && m + 8 <= m_end) *(u32x4*)to = u32x4{0u, 0u, 0u, 0u};
      else
        for (int e = 0; e < 8; ++e)
          if (m + e >= r.lo && m + e < m_end) to[e] = (_Float16)0.f;
    }
  }
  __syncthreads();

  floatx16 acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int x = 0; x < 16; ++x) acc[i][j][x] = 0.f;

  // operands of one step
  struct Step { int4v a[MB], b[NB]; int sa[MB], sb; };
  uint32_t tok[MB];                       // tokens behind M: the last one (their sums are not stored)
#pragma unroll
  for (int i = 0; i < MB; ++i) tok[i] = (uint32_t)min(m0 + (wm * MB + i) * 32 + (lane & 31), g.M - 1);
  const int nb0 = sub * CB + wn * NB;     // first column block of the wave
  const uint8_t* wv = g.vals + ((size_t)tile.step0 * GB + nb0) * 1024 + lane * 16;
  const uint8_t* ws = g.wscale + ((size_t)tile.step0 * 64 + lane) * GB;
  const uint32_t ldq = (uint32_t)g.ldq;
  const int half = lane >> 5;
  auto load = [&](int s, Step& x) {
    const uint32_t b = list[2 * s + half];
    const uint8_t* q = g.Q + (uint64_t)b * ldq * 16u;
    const uint8_t* sc = g.S + (uint64_t)b * ldq;
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      x.a[i] = *(const int4v*)(q + tok[i] * 16u);
      x.sa[i] = sc[tok[i]];
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) x.b[j] = *(const int4v*)(wv + (size_t)s * (GB * 1024) + j * 1024);
    if constexpr (GB == 4) x.sb = *(const int*)(ws + (size_t)s * 256);
    else x.sb = *(const uint16_t*)(ws + (size_t)s * 128);
  };
  auto multiply = [&](const Step& x) {
    const int sb = (int)((uint32_t)x.sb >> (8 * nb0));
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      acc[i][0] = mfma4<0>(x.a[i], x.b[0], acc[i][0], x.sa[i], sb);
      if constexpr (NB > 1) acc[i][1] = mfma4<1>(x.a[i], x.b[1], acc[i][1], x.sa[i], sb);
      if constexpr (NB > 2) acc[i][2] = mfma4<2>(x.a[i], x.b[2], acc[i][2], x.sa[i], sb);
      if constexpr (NB > 3) acc[i][3] = mfma4<3>(x.a[i], x.b[3], acc[i][3], x.sa[i], sb);
    }
  };

  // D steps under way: the wave's steps are wk, wk + WK, .. (n of them)
  const int n = (ns - wk + WK - 1) / WK;
  if (n > 0) {
    Step st[D];
#pragma unroll
    for (int d = 0; d < D; ++d) load(wk + min(d, n - 1) * WK, st[d]);
    int i = 0;
    for (; i + 2 * D <= n; i += D)
#pragma unroll
      for (int d = 0; d < D; ++d) {
        multiply(st[d]);
        load(wk + (i + D + d) * WK, st[d]);
      }
#pragma unroll
    for (int d = 0; d < D; ++d)
      if (i + d < n) {
        multiply(st[d]);
        if (i + D + d < n) load(wk + (i + D + d) * WK, st[d]);
      }
    i += D;
#pragma unroll
    for (int d = 0; d < D; ++d)
      if (i + d < n) multiply(st[d]);
  }

  // acc[i][j][x] is token 8 (x / 4) + 4 (lane / 32) + x % 4, column lane % 32 of block (i, j)
  char* mine = stage + wave * AREA;
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int row = j * 32 + (lane & 31), m = i * 32 + 8 * x + 4 * half;
        if constexpr (WK == 1) {
          half4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = (_Float16)acc[i][j][4 * x + e];
          *(half4*)(mine + row * PITCH + m * 2) = v;
        } else {
          floatx4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = acc[i][j][4 * x + e];
          *(floatx4*)(mine + row * PITCH + m * 4) = v;
        }
      }
  __syncthreads();
  auto store = [&](int col, int m, half8 v) {
    if (col < 0) return;
    _Float16* to = g.C + (size_t)(col - col_base) * g.ldc + m;
    if (m >= r.lo && m + 8 <= m_end) __builtin_nontemporal_store(v, (half8*)to);
    else
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (m + e >= r.lo && m + e < m_end) to[e] = v[e];
  };
  const int32_t* cols = g.col_idx + (size_t)t * (GB * 32) + sub * CB * 32;
  if constexpr (WK == 1) {
    constexpr int PPR = 4 * MB;           // pieces of 8 tokens per row of the wave's tile
#pragma unroll
    for (int i = 0; i < NB * 32 * PPR / 64; ++i) {
      const int p = i * 64 + lane, row = p / PPR, m = m0 + wm * MB * 32 + p % PPR * 8;
      store(cols[wn * NB * 32 + row], m, *(const half8*)(mine + row * PITCH + p % PPR * 16));
    }
  } else {
    for (int p = tid; p < WM * WN * 128; p += NT) {        // 32 rows x 4 pieces per block of C
      const int w = p / 128, row = p / 4 % 32, piece = p % 4;
      float s[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] = 0.f;
      for (int k = 0; k < WK; ++k) {
        const char* at = stage + (k * WM * WN + w) * AREA + row * PITCH + piece * 32;
        const floatx4 lo = *(const floatx4*)at, hi = *(const floatx4*)(at + 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) { s[e] += lo[e]; s[4 + e] += hi[e]; }
      }
      half8 v;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (_Float16)s[e];
      store(cols[(w / WM) * 32 + row], m0 + (w % WM) * 32 + piece * 8, v);
    }
  }
}

template <int GB, int MB, int NB, int WM, int WN, int WK, int D>
static hipError_t launch_mx4(GemmMx4Args g, hipStream_t stream) {
  constexpr int TM = 32 * MB * WM, SUB = GB / (NB * WN);
  int64_t mtiles = ((int64_t)g.M + TM - 1) / TM;
  if (g.offsets) {                        // most tiles that ranges of M tokens together can be cut into
    const int64_t met = g.n_members < g.M ? g.n_members : g.M;
    mtiles = ((int64_t)g.M + met * (TM + 6)) / TM;
  }
  const int64_t grid = mtiles * g.n_tiles * SUB;
  if (grid * (64 * WM * WN * WK) > 0xffffffffll) return hipErrorInvalidValue;
  g.n_mtiles = (int)mtiles;
  return launch_kernel(gemm_mx4_kernel<GB, MB, NB, WM, WN, WK, D>, dim3((unsigned)grid), dim3(64 * WM * WN * WK), stream, g);
}

template <int GB>
static hipError_t dispatch_mx4(const GemmMx4Args& g, hipStream_t stream) {
  // few tokens (per expert): 32 x 32 tiles whose eight waves share out the steps
  const int64_t tokens = g.offsets ? (int64_t)g.M / g.n_members : g.M;
  if (tokens <= 64) return launch_mx4<GB, 1, 1, 1, 1, 8, 2>(g, stream);
  if constexpr (GB == 4) return launch_mx4<4, 2, 2, 2, 2, 1, 3>(g, stream);
  else return launch_mx4<2, 2, 1, 2, 2, 1, 3>(g, stream);
}

hipError_t launch_gemm_mx4(int G, GemmMx4Args g, hipStream_t stream) {
  return G == 128 ? dispatch_mx4<4>(g, stream) : dispatch_mx4<2>(g, stream);
}

}  // namespace twg
