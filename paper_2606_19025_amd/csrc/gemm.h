// Shared by the grouped-GEMM kernels (large bf16 tiles: gemm.hip, the others:
// gemm_tile.hip): the
// GEMM kinds, their arguments, the group table and the launch record.
#pragma once
#include <type_traits>

#include "common.h"

namespace moe {

// UP_FWD and DH_BWD are GU_FWD and DHH_BWD for the SiLU expert (one first
// projection W1 [H, d] instead of [Wg; Wu]).
// XE_*: the products of a linear head's cross entropy (xent.hip), one group of the tokens
// that count: logits to partial sums of exponentials, logits to their gradient dz, dz W and
// dz^T x.
enum GemmKind {
  GU_FWD = 0, DOWN_FWD = 1, DHH_BWD = 2, DX_BWD = 3, DWD = 4, DWGU = 5, UP_FWD = 6, DH_BWD = 7,
  XE_LSE = 8, XE_DZ = 9, XE_DX = 10, XE_DW = 11
};

template <int KIND>
struct Kind {
  // ragged in M (else in K)
  static constexpr bool MRAG = KIND <= DX_BWD || (KIND >= UP_FWD && KIND != XE_DW);
  static constexpr bool A_KC = MRAG;  // A contiguous along k
  // B contiguous along k
  static constexpr bool B_KC = KIND <= DOWN_FWD || KIND == UP_FWD || KIND == XE_LSE || KIND == XE_DZ;
  static constexpr bool XE = KIND >= XE_LSE;
};

// What the XE_* kinds take besides: rows are the tokens that count, columns a piece [v0, v0 + V)
// of the vocabulary.
struct XentArgs {
  const void* x_all;      // x itself, taken instead of the counted tokens' copy when all count
  const int32_t* label;   // per row
  const float* lse;       // per row (XE_DZ)
  const float* coef;      // per row: its upstream gradient (XE_DZ)
  const float* out;       // XE_DW: a factor of all of it
  float2* part;           // XE_LSE: [128-column (small tiles: half a tile's) piece][cap] (max, sum), base 2
  float* z_label;         // XE_LSE: per row, the label's logit
  int V, v0;
  float scale, z2;        // of the logits; 2 z_coef
  int out_bf16;           // XE_DW: C is bf16
  int lo;                 // XE_DZ, small tiles: dz's rounding errors go this many elements behind it (0: nowhere)
  int* done;              // XE_LSE: a counter to clear for the launch that follows
};

struct GemmArgs {
  const void* A;
  const void* B;
  void* C;
  const void* aux;  // gu, read by the DHH_BWD epilogue
  void* out2;       // h, written by the GU_FWD epilogue
  const int32_t* offsets;  // NULL: one group of all cap rows
  long lda, ldb, ldc;
  long b_gs, c_gs;  // per-group strides (elements) of B and C
  long c_split;     // stride (elements) between the split-K partial outputs
  int n_groups, cap, M, N, K, H, accumulate;
  int ksplit;       // K-ragged kinds: each group's rows split in ksplit parts (0 = 1)
  // DOWN_FWD and DX_BWD (bf16): the kernel may cut K into up to ksplit_max
  // parts (its choice from the device-side group sizes); part p's fp32
  // partial goes to part + p c_split ([cap, N] each) and the choice to
  // *ksplit_used, for splitk_rows_reduce_kernel.  ksplit_max <= 1: no split.
  int ksplit_max;
  float* part;
  int* ksplit_used;
  XentArgs xe;  // XE_*; XE_DX: its fp32 partials go to part, ksplit (>= 1) parts of K
};

DEVI int clamp_row(int v, int cap) { return v < 0 ? 0 : (v > cap ? cap : v); }

// Group table of one set, staged in LDS once per block: the group offsets
// clamped to [0, cap] (c), their running maximum (b: group g of an M-ragged
// kind is rows [b[g], b[g+1])) and the number of m-tiles before group g (p).
constexpr int kMaxGroups = 256;
struct GroupTable {
  int c[kMaxGroups + 1], b[kMaxGroups + 1], p[kMaxGroups + 1];
  int uneven;  // (ragged in K) a group's tiles take over 1.25 times the average
};

DEVI int wave_incl_max(int v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(v, o, 64);
    if (lane >= o) v = max(v, u);
  }
  return v;
}
DEVI int wave_incl_sum(int v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(v, o, 64);
    if (lane >= o) v += u;
  }
  return v;
}

// Fill t from set a for m-tiles of BM rows (one wave; n_groups <= kMaxGroups).
// tile_rows: what a tile of a set ragged in K takes besides its group's rows (fill
// and epilogue, in rows).  (Found here, where the rows are at hand: a pass of
// its own over the table was slower.)
template <int BM>
DEVI void build_group_table(const GemmArgs& a, GroupTable& t, int tile_rows) {
  const int lane = threadIdx.x & 63;
  const int ng = a.n_groups;
  int run = 0;
  for (int g0 = 0; g0 <= ng; g0 += 64) {
    const int g = g0 + lane;
    const int c = g > ng ? 0 : a.offsets ? clamp_row(a.offsets[g], a.cap) : g ? a.cap : 0;
    int m = wave_incl_max(g <= ng ? c : 0);
    if (g0 > 0) m = max(m, run);
    if (g <= ng) {
      t.c[g] = c;
      t.b[g] = m;
    }
    run = __shfl(m, 63, 64);
  }
  WAIT_LGKMCNT(0);  // the wave's own table writes (lanes read their neighbours')
  int acc = 0;
  bool uneven = false;
  const float most = 1.25f * ((float)run + (float)tile_rows * (float)ng);
  for (int g0 = 0; g0 <= ng; g0 += 64) {
    const int g = g0 + lane;
    const int rows = g < ng ? t.b[g + 1] - t.b[g] : 0;
    const int tiles = (rows + BM - 1) / BM;
    uneven = uneven || __ballot((float)(rows + tile_rows) * (float)ng > most) != 0;
    const int inc = wave_incl_sum(tiles);
    if (g <= ng) t.p[g] = acc + inc - tiles;
    acc += __shfl(inc, 63, 64);
  }
  t.uneven = uneven;  // (the same from every lane)
  WAIT_LGKMCNT(0);
}

// Kernel argument of the GEMM kernels: up to kMaxSets sets of groups, each of
// GEMM kind KA or KB (kind_b[s] != 0), whose tiles share one
// launch - the routed and the merged shared experts of one kind, and in the
// backward two independent kinds (dHh with dW_d, dX with dW_gu), so that
// tiles of different lengths fill the CUs together, keep the CUs out of step
// (their epilogue stores do not all fall at once) and fill each other's last
// round.
constexpr int kMaxSets = 4;
struct GemmLaunch {
  GemmArgs s[kMaxSets];
  int kind_b[kMaxSets];
  int n_sets;
  int* counters;  // non-null: per-XCD tile counters (zero at launch) for dynamic dealing
};

// Timing names of the launches; the small tiles' end in _tile.
#define MOE_GEMM_NAMES(S)                                                                     \
  {"gemm_gu_fwd" S, "gemm_down_fwd" S, "gemm_dhh_bwd" S, "gemm_dx_bwd" S, "gemm_dwd" S,       \
   "gemm_dwgu" S, "gemm_up_fwd" S, "gemm_dh_bwd" S, "gemm_dhh_dwd" S, "gemm_dh_dwd" S,        \
   "gemm_dx_dwgu" S, "gemm_xe_lse" S, "gemm_xe_dz" S, "gemm_xe_dx_dw" S}
constexpr const char* kGemmNames[] = MOE_GEMM_NAMES("");
constexpr const char* kTileNames[] = MOE_GEMM_NAMES("_tile");
constexpr int gemm_name_index(int ka, int kb) {
  return ka >= XE_LSE ? ka + 3 : ka == kb ? ka : ka == DHH_BWD ? 8 : ka == DH_BWD ? 9 : 10;
}

// Output tiles of the bf16 launches (fp32 ones choose by themselves).  TILE_32x64:
// launches of one kind only.
enum TileSize { TILE_256x256, TILE_64x128, TILE_64x64, TILE_32x64 };
// The small tiles (gemm_tile.hip): one launch over sets_a[0..na) of kind ka and
// sets_b[0..nb) of kind kb (kb == ka with nb = 0: one kind).
hipError_t run_gemm_tile(int bf16, int ka, int kb, const GemmArgs* sets_a, int na,
                         const GemmArgs* sets_b, int nb, TileSize size, hipStream_t s);

// The large tiles (gemm.hip) of the XE_* kinds, bf16: kind ka over one set, or XE_DX with XE_DW
// (b).  counters: zeroed, or NULL.
constexpr int kXcdCounters = 8;
hipError_t run_gemm_xent(int ka, const GemmArgs& a, const GemmArgs* b, int* counters, hipStream_t s);

// Which tiles a bf16 launch of XE_LSE or XE_DZ takes: what choose_tiles estimates for an up
// projection of its sizes; and which one of XE_DX with XE_DW, whose dx is cut into split[i] parts at
// 256 x 256, 64 x 128 and 64 x 64.
TileSize xent_logit_tiles(const GemmArgs& a);
TileSize xent_pair_tiles(const GemmArgs& dx, const GemmArgs& dw, const int* split);

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;

// Partial (max, sum of 2^(z - max)) of the 4 NJ logits z = acc * scale2 (base 2) that a lane holds of a
// row at columns c + 16 j + t, with those of the three lanes 16 apart that hold the row's others;
// whole: no column of the tile lies past the last, V - 1 (wave-uniform), else those are left out.
template <int NJ>
DEVI float2 xent_partial(f32x4_t (&acc)[NJ], float scale2, int c, int V, bool whole) {
  if (!whole) {
    const float none = scale2 < 0.0f ? INFINITY : -INFINITY;
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (c + 16 * j + t >= V) acc[j][t] = none;
  }
  float m = acc[0][0];
  if (scale2 >= 0.0f) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) m = fmaxf(fmaxf(fmaxf(fmaxf(m, acc[j][0]), acc[j][1]), acc[j][2]), acc[j][3]);
  } else {
#pragma unroll
    for (int j = 0; j < NJ; ++j) m = fminf(fminf(fminf(fminf(m, acc[j][0]), acc[j][1]), acc[j][2]), acc[j][3]);
  }
  m *= scale2;
  m = fmaxf(m, __shfl_xor(m, 16, 64));
  m = fmaxf(m, __shfl_xor(m, 32, 64));
  const float at = m == -INFINITY ? 0.0f : m;
  float s = 0.0f;
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int t = 0; t < 4; ++t) s += __builtin_amdgcn_exp2f(__builtin_fmaf(acc[j][t], scale2, -at));
  s += __shfl_xor(s, 16, 64);
  s += __shfl_xor(s, 32, 64);
  return float2{m, s};
}

// The same lane's logits become their gradients cf (zf exp(z - lse) - [column = y]), rounded by the
// caller; zeros from column V on.  lse2: of base 2; y: the label's column, or any other number.
template <int NJ>
DEVI void xent_gradient(f32x4_t (&acc)[NJ], float scale2, float lse2, float cf, float zf, int c, int y, int V,
                        bool whole) {
  const float k = cf * zf;
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int t = 0; t < 4; ++t)
      acc[j][t] = k * __builtin_amdgcn_exp2f(__builtin_fmaf(acc[j][t], scale2, -lse2));
  if (__ballot((unsigned)(y - c) < 16u * NJ)) {
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (y == c + 16 * j + t) acc[j][t] -= cf;
  }
  if (!whole) {
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (c + 16 * j + t >= V) acc[j][t] = 0.0f;
  }
}

}  // namespace moe
