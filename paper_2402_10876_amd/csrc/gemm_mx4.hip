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

// Sum over the lanes up to the own one: inside rows of 16 lanes, then the rows' totals handed on (no LDS).
__device__ __forceinline__ int prefix_sum(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);        // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);       // lane 15 of a row to the next row (rows 1 and 3)
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);       // lane 31 to rows 2 and 3
  return x;
}

// The tokens of M-tile mt when they are shared out by expert: expert e owns [offsets[e], offsets[e+1]) (cut to [0, M); an
// end in front of its start: none) in tiles of TM that start on a multiple of align_of(TM).  Every wave finds it by itself.
// Tiles of 64 tokens and more start on lines of C (8 experts, 8192 tokens x 1024 columns: 1.25 times the time of one range with starts on 16 bytes,
// 1.03 with lines), smaller ones on 16 bytes, so that an expert of few tokens has one tile.  A piece of 16 bytes that an expert owns
// in part is written in at most three stores (32 experts, 4000 tokens x 1024 columns 9.8 -> 9.1 us).
struct Range { int e, m0, lo, hi; };
constexpr int align_of(int TM) { return TM >= 64 ? 64 : 8; }
template <int TM>
__device__ __forceinline__ bool find_range(const GemmMx4Args& g, int mt, int lane, Range& r) {
  constexpr int MASK = ~(align_of(TM) - 1);
  int before = 0;
  for (int c = 0; c < g.n_members; c += 64) {
    const int e = c + lane;
    int a = 0, b = 0;
    if (e < g.n_members) {
      a = min(max(g.offsets[e], 0), g.M);
      b = min(max(g.offsets[e + 1], 0), g.M);
    }
    const int tiles = b > a ? (b - (a & MASK) + TM - 1) / TM : 0;
    const int incl = prefix_sum(tiles);
    const unsigned long long hit = __ballot(before + incl > mt);
    if (hit) {
      const int f = __ffsll((long long)hit) - 1;
      const int start = before + __builtin_amdgcn_readlane(incl - tiles, f);
      const int af = __builtin_amdgcn_readlane(a, f);
      r.e = c + f;
      r.m0 = (af & MASK) + (mt - start) * TM;
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
__global__ __launch_bounds__(64 * WM * WN * WK, (MB * NB == 8 ? 2 : 1)) void gemm_mx4_kernel(GemmMx4Args g) {
  constexpr int NT = 64 * WM * WN * WK;
  constexpr int TM = 32 * MB * WM, CB = NB * WN;            // tokens, column blocks of the workgroup
  constexpr int SUB = GB / CB;                              // workgroups per tile of columns
  static_assert(GB % CB == 0 && (WK == 1 || (MB == 1 && NB == 1)), "");
  // staged output: WK = 1 a wave's halves [n][m], else the waves' fp32 partial sums [wave][n][m]
  constexpr int PITCH = WK == 1 ? 32 * MB * 2 + 16 : 36 * 4;
  constexpr int AREA = 32 * NB * PITCH;
  // (the list of blocks lies in front of it: 256 x 128 tiles of four waves come twice into a CU's LDS without the 8 KiB
  // beside them, 12.9 against 15.8 us for 1024 x 4096, half, at M = 4096)
  constexpr int STAGE = WM * WN * WK * AREA;
  __shared__ __attribute__((aligned(16))) char stage[STAGE > MAX_BLOCKS * 2 ? STAGE : MAX_BLOCKS * 2];
  uint16_t* list = (uint16_t*)stage;
  constexpr int ZL = 64;                                    // pruned columns whose numbers are fetched with the list
  __shared__ int cols[CB * 32], zeros[ZL];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % WM, wn = wave / WM % WN, wk = wave / (WM * WN);
  const int nt = g.n_tiles * SUB;
  const int lid = xcd_remap(blockIdx.x, gridDim.x);
  const int mt = lid / nt;
  int t = (lid - mt * nt) / SUB;
  const int sub = (lid - mt * nt) % SUB;

  Range r{0, mt * TM, mt * TM, g.M};
  if (g.offsets) {
    if (!find_range<TM>(g, mt, lane, r)) return;
    t += r.e * g.n_tiles;
  }
  const int col_base = r.e * g.member_n;
  const int m0 = r.m0, m_end = min(r.hi, m0 + TM);
  // the tile's record, its list of blocks (whatever is in use of it) and its columns in one round trip
  const Mx4Tile tile = g.tiles[t];
  const uint16_t* blocks = g.blocks + (size_t)t * g.list_len;
  const int32_t* col_idx = g.col_idx + (size_t)t * (GB * 32) + sub * CB * 32;
  constexpr int CPT = (CB * 32 + NT - 1) / NT;
  const u32x4 l0 = tid * 8 < g.list_len ? *(const u32x4*)(blocks + tid * 8) : u32x4{0u, 0u, 0u, 0u};
  int c0[CPT];
#pragma unroll
  for (int i = 0; i < CPT; ++i) c0[i] = col_idx[min(tid + i * NT, CB * 32 - 1)];
  if (tid * 8 < g.list_len) *(u32x4*)(list + tid * 8) = l0;
#pragma unroll
  for (int i = 0; i < CPT; ++i)
    if (tid + i * NT < CB * 32) cols[tid + i * NT] = c0[i];
  const int z0 = tile.zero_beg + (int)((int64_t)(tile.zero_end - tile.zero_beg) * sub / SUB);
  const int nz = tile.zero_beg + (int)((int64_t)(tile.zero_end - tile.zero_beg) * (sub + 1) / SUB) - z0;
  if (tid < min(nz, ZL)) zeros[tid] = g.zero_cols[z0 + tid];
  for (int i = (NT + tid) * 8; i < g.list_len; i += NT * 8) *(u32x4*)(list + i) = *(const u32x4*)(blocks + i);
  const int ns = tile.steps;

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
  auto load_w = [&](int s, Step& x) {
#pragma unroll
    for (int j = 0; j < NB; ++j) x.b[j] = *(const int4v*)(wv + (size_t)s * (GB * 1024) + j * 1024);
    if constexpr (GB == 4) x.sb = *(const int*)(ws + (size_t)s * 256);
    else x.sb = *(const uint16_t*)(ws + (size_t)s * 128);
  };
  auto load_a = [&](int s, Step& x) {
    const uint32_t b = list[2 * s + half];
    const uint8_t* q = g.Q + (uint64_t)b * ldq * 16u;
    const uint8_t* sc = g.S + (uint64_t)b * ldq;
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      x.a[i] = *(const int4v*)(q + tok[i] * 16u);
      x.sa[i] = sc[tok[i]];
    }
  };
  auto load = [&](int s, Step& x) { load_a(s, x); load_w(s, x); };
  auto multiply_row = [&](int i, const Step& x, int sb) {
    acc[i][0] = mfma4<0>(x.a[i], x.b[0], acc[i][0], x.sa[i], sb);
    if constexpr (NB > 1) acc[i][1] = mfma4<1>(x.a[i], x.b[1], acc[i][1], x.sa[i], sb);
    if constexpr (NB > 2) acc[i][2] = mfma4<2>(x.a[i], x.b[2], acc[i][2], x.sa[i], sb);
    if constexpr (NB > 3) acc[i][3] = mfma4<3>(x.a[i], x.b[3], acc[i][3], x.sa[i], sb);
  };
  auto multiply = [&](const Step& x) {
    const int sb = (int)((uint32_t)x.sb >> (8 * nb0));
#pragma unroll
    for (int i = 0; i < MB; ++i) multiply_row(i, x, sb);
  };

  // multiply and load in one, the loads in between the products: the order that a wave holds which is alone on its SIMD.  Left to
  // itself the compiler gathers the loads of all D steps behind their products and waits for all at once (4096 x 4096, M =
  // 8192, 82.3 against 78.3 us, half 49.3 against 46.4; shapes with more waves on a SIMD lose 1 to 5 % by it).
  constexpr bool HOLD = MB * NB == 16;
  auto multiply_load = [&](Step& x, int s) {
    const int sb = (int)((uint32_t)x.sb >> (8 * nb0));
    const uint32_t b = list[2 * s + half];
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      multiply_row(i, x, sb);
      __builtin_amdgcn_sched_barrier(0);
      x.a[i] = *(const int4v*)(g.Q + (uint64_t)b * ldq * 16u + tok[i] * 16u);
      x.sa[i] = g.S[(uint64_t)b * ldq + tok[i]];
      __builtin_amdgcn_sched_barrier(0);
    }
    load_w(s, x);
    __builtin_amdgcn_sched_barrier(0);
  };

  // D steps under way: the wave's steps are wk, wk + WK, .. (n of them)
  const int n = (ns - wk + WK - 1) / WK;
  Step st[D];
  if (n > 0) {
#pragma unroll
    for (int d = 0; d < D; ++d) load_w(wk + min(d, n - 1) * WK, st[d]);
  }
  __syncthreads();
  if (n > 0) {
#pragma unroll
    for (int d = 0; d < D; ++d) load_a(wk + min(d, n - 1) * WK, st[d]);
    int i = 0;
    for (; i + 2 * D <= n; i += D)
#pragma unroll
      for (int d = 0; d < D; ++d) {
        if constexpr (HOLD) {
          multiply_load(st[d], wk + (i + D + d) * WK);
        } else {
          multiply(st[d]);
          load(wk + (i + D + d) * WK, st[d]);
        }
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

  const bool lines = TM >= 64 && r.lo == m0 && m_end == m0 + TM;        // whole lines of C
  auto store = [&](int col, int m, half8 v) {
    if (col < 0) return;
    _Float16* to = g.C + (size_t)(col - col_base) * g.ldc + m;
    if (m >= r.lo && m + 8 <= m_end) {
      if (lines) __builtin_nontemporal_store(v, (half8*)to);
      else *(half8*)to = v;
    } else if (m + 8 <= m_end) {
      if (m + 8 > r.lo) store_back(to, v, 8 - (r.lo & 7));
    } else if (m >= r.lo) {
      if (m < m_end) store_front(to, v, m_end & 7);
    } else
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (m + e >= r.lo && m + e < m_end) to[e] = v[e];
  };
  // the workgroup's share of the pruned columns: 0 (here, where no load waits behind these stores)
  const int p0 = (r.lo - m0) >> 3, np = ((m_end - m0 + 7) >> 3) - p0;
  for (int i = tid; i < nz * np; i += NT) {
    const int z = i / np;
    store(z < ZL ? zeros[z] : g.zero_cols[z0 + z], m0 + (p0 + i - z * np) * 8, half8{0, 0, 0, 0, 0, 0, 0, 0});
  }

  __syncthreads();                          // everybody is done with the list
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
    mtiles = ((int64_t)g.M + met * (TM - 1 + align_of(TM) - 1)) / TM;
  }
  const int64_t grid = mtiles * g.n_tiles * SUB;
  if (grid * (64 * WM * WN * WK) > 0xffffffffll) return hipErrorInvalidValue;
  return launch_kernel(gemm_mx4_kernel<GB, MB, NB, WM, WN, WK, D>, dim3((unsigned)grid), dim3(64 * WM * WN * WK), stream, g);
}

// Tile shapes, tokens x columns (waves), us per launch in a captured stream of launches, operands from HBM, K x N and
// the share of the blocks kept:
//   R 512 x 128 (4)   wave tiles of 128 x 128: one read of the caches per 16 matrix instructions
//   Q 256 x 128 (4)   wave tiles of 64 x 128
//   V  64 x 128 (1)   W  64 x 64 (1)   U  32 x 64 (1)   waves on their own: none waits for another
//   P 128 x 128 (4)   wave tiles of 64 x 64
//   S  32 x 32 (4 on shares of the list, 2 of a short one)   S2 64 x 32 (2 x 4)
// Tiles below are counted as 64 x 128, steps are of the longest list, half of the blocks kept unless said otherwise.
// S, S2: lists shared among waves, where single waves would leave CUs idle.  Up to 12 steps S (two waves), to 1280 workgroups, with 4 steps or
// tiles of 64 columns to 1024; S / U: 1024 x 1024, 8 steps, M = 1024 3.95 / 4.45, M = 1280 4.26 / 4.65, M = 1536 4.81 / 4.78; a quarter, 4 steps, M = 1024 3.53 /
// 3.60, M = 1280 4.04 / 3.77; 1024 x 4096, 8 steps, M = 320 5.0 / 5.3, M = 384 5.7 / 5.4; S2 3.8 where S takes 3.4 (M = 512).  From 16 steps on
// S2 to two workgroups a CU (128 tiles), S while it has one: S / S2 / U 2048 x 1024, M = 192 3.8 / 3.9 / 5.1, M = 1024 5.3 / 5.6 / 5.5, M = 1152
// 5.6 / 7.1 / 5.7; 4096 x 4096, M = 128 6.0 / 5.2 / 7.3, M = 256 8.7 / 7.2 / 9.1; 8192 x 1024, M = 192 5.5 / 6.1 / 10.5, M = 1024 10.6 / 9.7 / 11.3,
// M = 1152 11.9 / 12.3 / 11.3.  Shares of S: two, four with 4 steps under way, four with 8: 1024 x 4096, 8 steps, M = 1 3.0, 3.2, 3.5; 2048 x
// 1024, 8 experts (16 steps), M = 256 5.1, 5.3, 5.9; 1536 x 672 (about 14), M = 359 3.8, 3.6; 4096 x 4096 (32), M = 32 4.1, 3.75, 3.6, all (64)
// 6.4, 5.4, 4.8.
// R: one workgroup a CU, so the last round has to be worth it.  One round from 384 tiles of 256 rows and 32 steps on: 4096 x 4096, M = 4096 R
// 25.6, Q 29.0, V 29.1, M = 2560 23.1, 24.2, 21.3; 16 steps R 18.4, Q 18.5.  More rounds, 16 steps: 2048 x 4096, M = 4352 (32 tiles past the
// first) R 28.6, Q 25.2, M = 5000 (128) 30.5, 29.7, M = 5400 (192) 30.1, 29.7, M = 5900 (256) 33.2, 35.0, M = 8704 (64 past the second) 43.5,
// 40.7, M = 9216 (128) 43.4, 42.2, M = 10000 (256) 48.1, 53.4; 32 steps: 4096 x 4096, M = 4600 (64) 41.1, 38.5, M = 5000 (128) 42.7, 42.8, M =
// 8704 (64 past the second) 63.6, 65.5; 64 steps: M = 4352 (32) 62, 64, M = 8192 77, 95; 8192 cubed R 263.
// Q, V, W by rounds: a CU holds 12 waves of W (1536 tiles), 8 of V or 2 workgroups of Q (2048).  1024 x 4096, a tenth of the columns
// pruned: M = 3100 (1421 tiles) W 12.1, V 12.7, Q 12.9; M = 4096 (1856) 15.0, 13.6, 13.3; M = 5000 (2291) 20.1, 20.2, 19.8; M = 6000
// (2726) 27.8, 23.8, 21.9; nothing pruned M = 4992 (2496) W 19.0, Q 19.1, M = 5120 (2560) 19.8, 19.2; a quarter, M = 5000 14.3, 16.4, 16.3.
// V from 16 steps on: 2048 x 4096, M = 2304 (1152) W 13.3, V 13.6, M = 2432 (1216) 14.0, 13.7, M = 3072 (1536) 18.1, 15.8.
// P in one round, above 160 tiles of 128 rows, up to 28 steps above 192: 4096 x 4096, M = 600 (160) P 10.2, U 10.3, M = 700 (192) 10.5, 11.3, M = 1024 (256) 11.3,
// 13.2; 16 steps 7.5, 7.3; 7.8, 7.8; 8.3, 8.8; 20 steps 2041 x 3616, M = 822 (182) 9.6, 9.2; 8192 x 4096, M = 700 16.3, 18.2; short lists 1024 x 4096, M = 1024 6.9, U 6.8.
// W from 640 tiles, from 24 steps on from the end of U's two waves a SIMD (512): 1024 x 1024, M = 4608 (576) W 7.1, U 6.8, M = 5120 (640) 7.25, 7.2,
// M = 5632 7.6, 7.7; 2048 x 4096, M = 1088 (544) 9.4, 9.6; 4096 x 4096 13.3, 15.0.
// By expert, where ranges end inside tiles (tiles: those of M tokens and one more for every expert).  S / U, 8 steps, to 1280 workgroups as above: 1024
// x 1024, 8 experts, M = 800 (264 of 32 rows) 4.7 / 5.3, M = 1200 (360) 5.4 / 5.5, 32 experts, M = 700 (424) 6.7 / 6.7, 1024 x 2048, 8 experts, M
// = 800 (528) 6.3 / 6.2; 16 steps, to 1024: 4 experts, M = 900 (256) 5.8 / 6.3, 32 experts, M = 300 (328) 8.4 / 8.1.  V, 8 steps, above 1240
// tiles: 1024 x 2048, 4 experts, M = 4600 (1200) W 11.0, V 12.0, 16 experts, M = 4000 (1248) 15.1, 14.3, 8 experts of 1024 columns, M = 11500 (1496)
// 17.2, 15.0; 4 steps, above 1536: 96 x 1024, 8 experts, M = 11000 (1432) 8.8, 10.0, M =
// 12500 (1624) 11.6, 10.5; 16 steps, above 1100: 8 experts, M = 8192 (1088) 15.8, 16.3, M = 9000 (1184) 18.6, 17.2, 32 experts, M = 7000 (1128) 20.4,
// 19.0; Q 0.7 to 2 us more than V.  W from 192 tokens an expert on: 8 experts, M = 6000 W 8.8, U 9.4, 16 experts, M = 5000 (16 steps) 13.2,
// 13.8, 32 experts, M = 6000 13.4, 12.4, M = 7000 14.4, 14.1; 256 experts, M = 16384 V 48, U 50, W 55.
// Tiles of 64 columns: no V by expert (512 x 3200, 5 experts, M = 6449 W 19.3, V 20.5; with 1024 x 4096 W 37, V 36), and U by two waves of
// 32 x 32 up to 600 tiles of 32 rows and short lists (640 x 512, M = 4000 (500) 4.3 against 4.4, M = 5000 (628) 4.9 and 5.0, M = 7000 (876) 5.7 and
// 5.3; 2048 x 1024, 8 experts, M = 2048, 16 steps 7.6 against 7.1).
template <int GB>
static hipError_t dispatch_mx4(const GemmMx4Args& g, hipStream_t stream) {
  const int64_t M = g.M, n = ((int64_t)g.n_tiles * GB + 3) / 4;        // column tiles of 128
  const int steps = g.list_len / 2;
  enum { R, Q, P, V, W, U, S, S2 } shape;
  int64_t tiles32;
  const int short_most = GB == 4 && steps > 4 && steps < 16 ? 320 : 256;
  if (g.offsets && M / g.n_members < 4096) {
    const int64_t met = g.n_members < M ? g.n_members : M, tiles64 = (M / 64 + met) * n;
    tiles32 = (M / 32 + met) * n;
    if (tiles32 <= short_most) shape = S;
    else if (GB == 4 && tiles64 > (steps >= 16 ? 1100 : steps > 4 ? 1240 : 1536)) shape = V;
    else shape = tiles64 >= 640 && M / g.n_members >= 192 ? W : U;
  } else {
    auto tiles = [&](int rows) { return (M + rows - 1) / rows * n; };
    tiles32 = tiles(32);
    const int64_t t256 = tiles(256), past = t256 % 512;      // past: tiles of R (two of these) in its last round
    const bool one_round = t256 <= 512;
    if (steps < 16 ? tiles32 <= short_most : tiles(64) <= 128) shape = steps < 16 || M <= 32 || tiles32 * 4 <= 256 ? S : S2;
    else if (t256 >= 384 && (one_round ? steps >= 32 : steps >= 64 || (steps >= 32 ? t256 >= 640 : steps >= 16 && (past == 0 || past > 192)))) shape = R;
    else if (tiles(64) > 2450 || (tiles(64) > 1536 && (tiles(64) <= 2048 || steps >= 16))) shape = Q;
    else if (tiles(64) >= 1200 && steps >= 16) shape = V;
    else if (steps >= 16 && tiles(128) > (steps >= 32 ? 160 : 192) && tiles(128) <= 256) shape = P;
    else shape = tiles(64) >= 640 || (tiles(64) > 512 && steps >= 24) ? W : U;
  }
  if (shape == S) {
    if (steps <= 12) return launch_mx4<GB, 1, 1, 1, 1, 2, 4>(g, stream);
    return steps <= 32 ? launch_mx4<GB, 1, 1, 1, 1, 4, 4>(g, stream) : launch_mx4<GB, 1, 1, 1, 1, 4, 8>(g, stream);
  }
  if (shape == S2) return launch_mx4<GB, 1, 1, 2, 1, 4, 4>(g, stream);
  if (GB == 2 && shape == U && tiles32 <= 600 && steps <= 12) return launch_mx4<2, 1, 1, 1, 2, 1, 4>(g, stream);
  if (shape == U) return launch_mx4<GB, 1, 2, 1, 1, 1, 4>(g, stream);
  if (shape == W) return launch_mx4<GB, 2, 2, 1, 1, 1, GB == 4 ? 2 : 3>(g, stream);
  if constexpr (GB == 4) {
    if (shape == R) return launch_mx4<4, 4, 4, 4, 1, 1, 3>(g, stream);
    if (shape == Q) return launch_mx4<4, 2, 4, 4, 1, 1, 2>(g, stream);
    if (shape == P) return launch_mx4<4, 2, 2, 2, 2, 1, 4>(g, stream);
    return launch_mx4<4, 2, 4, 1, 1, 1, 2>(g, stream);
  } else {      // tiles of 64 columns: R and Q 512 x 64 (4 waves), P 256 x 64 (4), V 128 x 64 (1)
    if (shape == R || shape == Q) return launch_mx4<2, 4, 2, 4, 1, 1, 2>(g, stream);
    if (shape == P) return launch_mx4<2, 2, 2, 4, 1, 1, 4>(g, stream);
    return launch_mx4<2, 4, 2, 1, 1, 1, 2>(g, stream);
  }
}

hipError_t launch_gemm_mx4(int G, GemmMx4Args g, hipStream_t stream) {
  return G == 128 ? dispatch_mx4<4>(g, stream) : dispatch_mx4<2>(g, stream);
}

}  // namespace twg
