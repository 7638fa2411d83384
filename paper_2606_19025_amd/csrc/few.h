// The whole MoE layer for a few tokens (T <= 64): evaluation and generation.
//
//   z = (x Wr^T + b) / tau, top-k, gates           (as the router, to the bit)
//   h_tj = s_tj act(Wgu_e x_t)                      for each resident route (t, j) to expert e
//   y_t  = sum_j Wd_e h_tj + Wd_s act(Wgu_s x_t)    (s: the shared experts, gate 1)
//
// Bound by the weights' bytes: every active expert's are read once, for a handful of tokens each;
// those of an expert with more tokens than a pass holds, and the shared experts', once per pass:
// MXFP4 ceil(T / 8) passes past 8 tokens, bf16 two past 48 tokens, fp32 two past 32 (experts with
// up to 16 tokens: one).  An expert's pass without tokens is not skipped.
// Three launches: the logits (few_logits_*), the first projections (few_gu_kernel) and the
// second ones with the sum over experts (few_down_kernel).  No rows are moved: the weights
// are the matrix instruction's first operand (16 rows of an expert's matrix) and the tokens
// its second (16 columns).  The gate is in h, so that the second projections are plain sums.
// (The order of k within a matrix instruction is free as long as both operands have the same.)
//
// Measured (d = 2048, H = 1408, 64 experts, k = 6, shared 2816): one token, bf16, 5 + 20 + 15 us
// (the weights at 4.6 and 3.1 TB/s); 48 tokens on 16 resident experts 6 + 48 + 28; 16 tokens
// on 32 experts in MXFP4 5 + 31 + 25.  Some 130 MB of weights, which calls on the same ones may find
// in the last-level cache (256 MB); six layers in turn, other tokens each time: one token 41 us a
// call against 37, the 16 tokens 72 against 68.
// MXFP4, all 32 experts at hand, by tokens (event times of the projections, us): 1 16 + 14, 4 26 + 21,
// 8 30 + 25, 16 37 + 31, 24 43 + 36, 33 58 + 47, 48 110 + 89, 64 183 + 147.
#pragma once
#include <type_traits>

#include "kernels.h"
#include "mx.h"
#include "route_select.h"
#include "timing.h"

namespace moe {

constexpr int FEW_T = kFewTokens;  // tokens at most
constexpr int FEW_K = RT_KSEL;     // routes of a token at most

struct FewArgs {
  const void* x;
  const void* w_router;
  const float* bias;
  const uint8_t* resident;
  const void *wgu, *wd, *sgu, *sd;              // experts' weights (or codes), routed and shared
  const uint8_t *wgu_s, *wd_s, *sgu_s, *sd_s;   // and MXFP4 scales
  float* logits;
  int32_t* idx;
  float* tw;
  int32_t* local;
  void* y;
  // workspace
  int32_t* w_local;  // [T k]
  void* h;         // [T k, H]: rows of resident routes
  void* hs;        // [T, Hs]
  int T, d, E, k, E_r, H, Hs, gate;
  float inv_tau;
};

namespace {

// ------------------------------------------------------------------ routes
// The block's tables: each route's gate and local expert, and the experts that any token is
// routed to.
struct FewTables {
  float gate[FEW_T * FEW_K];
  int16_t local[FEW_T * FEW_K];
  int16_t expert[256];        // active expert -> local id
  int slot[256];              // tokens of a local expert
  int lmap[256];
  int n_class[3];             // experts with few tokens, more, many (few_active)
};

// Top-k and gates of token t, by 16 lanes (the router's selection on logits in
// global memory): lane s of a group holds the experts s, s + 16, ... in v[].
template <int NE>
DEVI void few_logits_of(const FewArgs& a, int t, float (&v)[NE]) {
  const int s = threadIdx.x & 15;
#pragma unroll
  for (int q = 0; q < NE; ++q) {
    const int e = q * 16 + s;
    v[q] = t < a.T && e < a.E ? sel_value(a.logits[(size_t)t * a.E + e]) : 0.f;
  }
}
template <int NE>
DEVI void few_select(const FewArgs& a, FewTables& tb, int t, const float (&v)[NE], bool publish) {
  const int lane = threadIdx.x & 63, s = lane & 15;
  const bool has = t < a.T;
  uint64_t cand[NE];
#pragma unroll
  for (int q = 0; q < NE; ++q) {
    const int e = q * 16 + s;
    cand[q] = has && e < a.E ? ((uint64_t)sel_key(v[q]) << 32) | (uint32_t)~e : 0ull;
  }
  int my_id = 0;
  float my_z = 0.f;
  for (int j = 0; j < a.k; ++j) {
    uint64_t m = 0ull;
#pragma unroll
    for (int q = 0; q < NE; ++q) m = max64(cand[q], m);
    m = row16_max64(m);
#pragma unroll
    for (int q = 0; q < NE; ++q)
      if (cand[q] == m) cand[q] = 0ull;
    if (s == j) {
      my_id = (int)~(uint32_t)m;
      const uint32_t key = (uint32_t)(m >> 32);
      my_z = __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
    }
  }
  const float zmax = __shfl(my_z, lane & 48, 64);
  float denom = 1.f;
  if (a.gate == MOE_GATE_SOFTMAX_TOPK || a.gate == MOE_GATE_SOFTMAX) {
    float acc = 0.f;
    if (a.gate == MOE_GATE_SOFTMAX_TOPK) {
      if (s < a.k) acc = expf(my_z - zmax);
    } else {
#pragma unroll
      for (int q = 0; q < NE; ++q)
        if (q * 16 + s < a.E) acc += expf(v[q] - zmax);
    }
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) acc += __shfl_xor(acc, o, 64);
    denom = acc;
  }
  if (s < a.k && has) {
    const float g = a.gate == MOE_GATE_SIGMOID ? sigmoid_f(my_z) : expf(my_z - zmax) / denom;
    const int o = t * a.k + s;
    tb.gate[o] = g;
    tb.local[o] = (int16_t)my_id;  // (few_localise makes it the local id)
    if (publish) {
      if (a.idx) a.idx[o] = my_id;
      if (a.tw) a.tw[o] = g;
    }
  }
}

// All tokens' selections by the WAVES waves of a block, every wave's logits loaded first.
template <int WAVES, int NE>
DEVI void few_select_all(const FewArgs& a, FewTables& tb, bool publish) {
  constexpr int P = FEW_T / (4 * WAVES);
  const int t = (threadIdx.x >> 6) * 4 + ((threadIdx.x & 63) >> 4);
  float v[P][NE];
#pragma unroll
  for (int p = 0; p < P; ++p) few_logits_of<NE>(a, t + p * 4 * WAVES, v[p]);
#pragma unroll
  for (int p = 0; p < P; ++p)
    if ((t & ~3) + p * 4 * WAVES < a.T) few_select<NE>(a, tb, t + p * 4 * WAVES, v[p], publish);
}

// Local ids of the routes' experts, or -1, from lmap[].
DEVI void few_localise(const FewArgs& a, FewTables& tb, bool publish) {
  for (int i = threadIdx.x; i < a.T * a.k; i += blockDim.x) {
    const int m = tb.lmap[tb.local[i]];
    // (a resident set larger than E_r says: its last experts are ghosts here)
    const int l = m < a.E_r ? m : -1;
    tb.local[i] = (int16_t)l;
    if (publish) {
      a.w_local[i] = l;
      if (a.local) a.local[i] = l;
    }
  }
}

// The active experts by their number of tokens (up to Q, up to M, more), each class in
// ascending order.  All threads call it, with slot[] zero and the routes in local[]; it
// ends with a barrier.
template <int Q, int M>
DEVI void few_active(const FewArgs& a, FewTables& tb) {
  for (int i = threadIdx.x; i < a.T * a.k; i += blockDim.x)
    if (tb.local[i] >= 0) atomicAdd(&tb.slot[tb.local[i]], 1);
  __syncthreads();
  if (threadIdx.x < 64) {
    const int lane = threadIdx.x;
    int n = 0;
    for (int cl = 0; cl < 3; ++cl) {
      const int n0 = n;
      for (int r0 = 0; r0 < a.E_r; r0 += 64) {
        const int r = r0 + lane;
        const int c = r < a.E_r ? tb.slot[r] : 0;
        const bool on = c > 0 && (c <= Q ? 0 : c <= M ? 1 : 2) == cl;
        const uint64_t m = __ballot(on);
        if (on) tb.expert[n + __popcll(m & ((1ull << lane) - 1ull))] = (int16_t)r;
        n += __popcll(m);
      }
      if (lane == 0) tb.n_class[cl] = n - n0;
    }
  }
  __syncthreads();
}

// Route (t k + j) of token t to local expert r, or -1.
DEVI int route_to(const FewArgs& a, const FewTables& tb, int t, int r) {
  int p = -1;
  if (t < a.T)
    for (int j = 0; j < a.k; ++j)
      if (tb.local[t * a.k + j] == r) p = t * a.k + j;
  return p;
}

// ------------------------------------------------------------------ operands
// One step of a wave: tiles of 16 weight rows and of 16 tokens by KS of k, brought to the
// wave's own ring in LDS by DMA, whole row pieces of 128 (weights) and XROW (activations)
// bytes, and read from there as operands: lane (r, q) = (lane % 16, lane / 16) holds row r.
//   bf16   KS 64, two v_mfma_f32_16x16x32_bf16 per pair of tiles
//   fp32   KS 32, eight v_mfma_f32_16x16x4_f32
//   MXFP4  KS 256 (and eight scales per row), widened to bf16 (exactly, a value has two
//          significant bits): eight v_mfma_f32_16x16x32_bf16 on bf16 activations
// (Loaded in operand order instead, straight to registers, a load instruction touches 16
// rows and a CU's address unit was the bound: 2.3 to 3.1 TB/s over the GPU.  MXFP4 steps of
// 128 fetched each 128-byte line for its halves twice.)
// XF, XM: DMA parts of a tile of activations for experts with few tokens and with more: 8 and
// 16 tokens, MXFP4 4 and 8 (a whole tile would take half of a ring).
template <class E, bool MX> struct Fmt;
template <> struct Fmt<bf16_t, false> { static constexpr int KS = 64, XROW = 128, XF = 1, XM = 2; };
template <> struct Fmt<float, false> { static constexpr int KS = 32, XROW = 128, XF = 1, XM = 2; };
template <> struct Fmt<bf16_t, true> { static constexpr int KS = 256, XROW = 512, XF = 2, XM = 4; };

// 16 bytes per lane from base + off (base uniform) to LDS at lds + 16 lane.  The asm sets m0
// and leaves the one wait state an LDS DMA needs after it.
DEVI void few_dma16(uint64_t base, unsigned off, unsigned lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(lds)
               : "m0", "memory");
}
// 4 bytes per lane, to lds + 4 lane.
DEVI void few_dma4(uint64_t base, unsigned off, unsigned lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(off), "s"(base), "s"(lds)
               : "m0", "memory");
}
DEVI uint64_t uniform64(const void* p) {
  const uint64_t v = (uint64_t)(uintptr_t)p;
  const uint64_t lo = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)v);
  const uint64_t hi = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(v >> 32));
  return hi << 32 | lo;
}

// Row pieces of B bytes as a DMA instruction brings them: part p holds the rows
// p * RPI + lane / LPR of a tile, and 16-byte chunk c of row r sits at chunk c ^ swz(r), so
// that the 16 lanes of an operand read (16 rows, one chunk) are free of bank conflicts.
template <int B>
struct Piece {
  static constexpr int LPR = B / 16, RPI = 64 / LPR, PARTS = 16 / RPI;
  DEVI static int swz(int r) { return LPR == 8 ? (r >> 1) & 7 : r & 15; }
  DEVI static int row(int part) { return part * RPI + (int)(threadIdx.x & 63) / LPR; }
  DEVI static int chunk(int part) { return ((int)(threadIdx.x & 63) % LPR) ^ swz(row(part)); }
  DEVI static const char* at(const char* tile, int r, int c) { return tile + r * B + ((c ^ swz(r)) << 4); }
};

typedef __bf16 bf16x2_v __attribute__((ext_vector_type(2)));
DEVI bf16x8_t mx_widen8(unsigned c, float s) {
  const bf16x2_v a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0);
  const bf16x2_v b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1);
  const bf16x2_v d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2);
  const bf16x2_v e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3);
  const bf16x8_t v = {a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
  return v;
}

// Waves that stream weights in few_gu_kernel and few_down_kernel, whose blocks have a CU each.
// The second's steps are a quarter as long, so that it takes two waves per SIMD to keep the
// loads coming.
constexpr int FW = 4, FT = 64 * FW, DW = 8, DT = 64 * DW;
// Bytes of a wave's ring: what a CU's 160 KB leave beside the sums and tables.
constexpr int gu_ring(int tiles) { return (tiles <= 2 ? 28 : 26) * 1024; }
constexpr int down_ring(int NT) { return (NT == 1 ? 18 : NT == 2 ? 17 : NT == 3 ? 16 : 14) * 1024; }

// A wave's stream of steps: RT tiles of weights and N of activations each.  WP, XP: DMA parts
// of a tile of either (fewer than all where only its first rows count).
template <class E, bool MX, int RT, int N, int WP, int XP, int RING>
struct Stream {
  using F = Fmt<E, MX>;
  using PW = Piece<128>;
  using PX = Piece<F::XROW>;
  static constexpr int W_TILE = WP * 1024, X_TILE = XP * 1024, X_AT = RT * W_TILE, S_AT = X_AT + N * X_TILE;
  static constexpr int STAGE = S_AT + (MX ? 512 : 0);
  static constexpr int PER = RT * WP + N * XP + (MX ? 2 : 0);   // DMA instructions of a step
  static constexpr int D0 = RING / STAGE, D = D0 > 12 ? 12 : D0;  // steps in flight
  static constexpr int XN = F::XROW / 64;                        // a lane's 16-byte chunks of a tile of x
  static_assert(D >= 2 && D * PER <= 63, "a ring of two steps, counted by vmcnt");
  static_assert(!MX || RT <= 4, "a DMA instruction brings a word of scales for 64 rows");

  unsigned woff[WP], xoff[N][XP], soff;  // lane offsets
  char* ring;
  unsigned ring_lds;
  int K;

  DEVI Stream(char* wave_ring, int k) : soff(0), ring(wave_ring), K(k) {
    ring_lds = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(lds_void_t*)wave_ring);
  }
  // line: bytes of a weight row; rows: those of a tile that exist (16, or fewer)
  DEVI void weights(unsigned line, int rows) {
#pragma unroll
    for (int p = 0; p < WP; ++p) woff[p] = min(PW::row(p), rows - 1) * line + PW::chunk(p) * 16;
  }
  // the row of activations of each column of tile n, by column
  DEVI void column(int n, int row_of_lane16) {
#pragma unroll
    for (int p = 0; p < XP; ++p) {
      const int row = __shfl(row_of_lane16, PX::row(p), 64);
      xoff[n][p] = (unsigned)row * (unsigned)(K * sizeof(E)) + PX::chunk(p) * 16;
    }
  }

  // w[i], scales, x: uniform addresses of the tiles' first row at step 0.  K is a multiple of
  // 64, so only an MXFP4 step can be cut: its lanes past the row's end read the row's piece
  // from its start, and read() makes their weights zeros.
  DEVI void issue(int slot, int st, const uint64_t* w, uint64_t scales, uint64_t x) const {
    const unsigned at = ring_lds + slot * STAGE;
    const int rest = K - st * F::KS;
    const bool cut = MX && rest < F::KS;
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int p = 0; p < WP; ++p) {
        unsigned o = woff[p];
        if (cut && PW::chunk(p) * 32 >= rest) o -= PW::chunk(p) * 16;
        few_dma16(w[i] + (uint64_t)st * 128, o, at + i * W_TILE + p * 1024);
      }
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int p = 0; p < XP; ++p) {
        unsigned o = xoff[n][p];
        if (cut && PX::chunk(p) * 8 >= rest) o -= PX::chunk(p) * 16;
        few_dma16(x + (uint64_t)st * F::XROW, o, at + X_AT + n * X_TILE + p * 1024);
      }
    if constexpr (MX) {
      // (a row of scales is whole words: the second one may not be there)
      few_dma4(scales + (uint64_t)st * 8, soff, at + S_AT);
      few_dma4(scales + (uint64_t)st * 8 + (rest > 128 ? 4 : 0), soff, at + S_AT + 256);
    }
  }

  // Operands of one step, in registers (of tiles that are brought in part, the rows that are
  // there again).
  struct Frags {
    u32x4_t w[RT][2];
    u32x4_t x[N][XN];
    unsigned s[RT][2];
  };
  DEVI void read(Frags& f, int slot, int st) const {
    const char* at = ring + slot * STAGE;
    const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int p = 0; p < 2; ++p)
        f.w[i][p] = *reinterpret_cast<const u32x4_t*>(PW::at(at + i * W_TILE, r & (WP * PW::RPI - 1), 4 * p + q));
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int p = 0; p < XN; ++p)
        f.x[n][p] = *reinterpret_cast<const u32x4_t*>(
            PX::at(at + X_AT + n * X_TILE, r & (XP * PX::RPI - 1), MX ? 16 * (p >> 2) + 4 * q + (p & 3) : 4 * p + q));
    if constexpr (MX) {
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int p = 0; p < 2; ++p)
          f.s[i][p] = *reinterpret_cast<const unsigned*>(at + S_AT + p * 256 + (16 * i + r) * 4) >> (8 * q) & 255u;
      const int rest = K - st * F::KS;
      if (rest < F::KS)
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
          for (int p = 0; p < 2; ++p)
            if (128 * p + 32 * q >= rest) f.w[i][p] = u32x4_t{0u, 0u, 0u, 0u};
      // (and the activations: 0 times an infinity that is read again is not 0)
      if (rest < F::KS)
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
          for (int p = 0; p < XN; ++p)
            if (128 * (p >> 2) + 32 * q >= rest) f.x[n][p] = u32x4_t{0u, 0u, 0u, 0u};
    }
  }
  DEVI static void mma(const Frags& f, f32x4_t (&acc)[RT][N]) {
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        if constexpr (MX) {
          const float s = mx_scale_f32(f.s[i][p]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bf16x8_t w = mx_widen8(f.w[i][p][e], s);
#pragma unroll
            for (int n = 0; n < N; ++n)
              acc[i][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                  w, __builtin_bit_cast(bf16x8_t, f.x[n][4 * p + e]), acc[i][n], 0, 0, 0);
          }
        } else {
#pragma unroll
          for (int n = 0; n < N; ++n) {
            if constexpr (sizeof(E) == 2) {
              acc[i][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                  __builtin_bit_cast(bf16x8_t, f.w[i][p]), __builtin_bit_cast(bf16x8_t, f.x[n][p]), acc[i][n], 0, 0, 0);
            } else {
              const f32x4_t a = __builtin_bit_cast(f32x4_t, f.w[i][p]), b = __builtin_bit_cast(f32x4_t, f.x[n][p]);
#pragma unroll
              for (int e = 0; e < 4; ++e)
                acc[i][n] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], acc[i][n], 0, 0, 0);
            }
          }
        }
      }
  }
};

// How a class of experts is taken: N tiles of XP DMA parts at a time; COMPACT: the expert's
// tokens moved to the front of one tile, otherwise all T tokens in as many passes over the weights
// as they need (most: MOST).  CT: columns of a tile that are used.
template <class E, bool MX, int N_, int XP_, int MOST_, bool COMPACT_>
struct Class {
  static constexpr int N = N_, XP = XP_, MOST = MOST_, CT = XP_ * Piece<Fmt<E, MX>::XROW>::RPI;
  static constexpr bool COMPACT = COMPACT_;
  DEVI static int passes(int T) { return MOST == 1 ? 1 : ceil_div(T, N * CT); }
};
// Few tokens, more in one compact tile, any number (in passes over the weights).
template <class E, bool MX, int NT, int NP>
struct Classes {
  using F = Fmt<E, MX>;
  typedef Class<E, MX, 1, F::XF, 1, true> Few;
  typedef Class<E, MX, 1, F::XM, 1, true> More;
  typedef Class<E, MX, NP, F::XM, (16 * NT + NP * More::CT - 1) / (NP * More::CT), false> All;
};

// Row of activations of each column of a wave's tiles of class C, from my_row (lane l: token
// l's, or -1): the column's token t and its row, -1 for none.  Compact: the tokens that have
// a row are moved to the front; otherwise pass p takes the tokens from p N CT on.
template <class C>
struct Cols {
  int t[C::N], row[C::N];
  DEVI Cols(int my_row, int pass) {
    const int lane = threadIdx.x & 63, l16 = lane & 15;
    int who = lane;
    if constexpr (C::COMPACT) {
      const uint64_t on = __ballot(my_row >= 0), below = (1ull << lane) - 1ull;
      const int to = my_row >= 0 ? __popcll(on & below) : __popcll(on) + __popcll(~on & below);
      who = __builtin_amdgcn_ds_permute(to * 4, lane);
    }
#pragma unroll
    for (int n = 0; n < C::N; ++n) {
      const int at = (pass * C::N + n) * C::CT + l16;
      t[n] = __shfl(who, at & 63, 64);
      const int r = __shfl(my_row, t[n], 64);
      row[n] = l16 < C::CT && at < 64 ? r : -1;
    }
  }
};

// Tiles that a pass over an expert's weights takes of a batch's NT, where tokens are many.
constexpr int gu_tiles(bool MX, int NT) { return MX ? 1 : NT == 4 ? 2 : NT; }
constexpr int down_tiles(bool MX, int NT) { return MX ? 1 : NT > 3 ? 2 : NT; }

// ------------------------------------------------------------------ first projections
// An item is 16 hidden units of one expert (for SwiGLU as many rows of W_g and of W_u).  Four
// waves of the block stream it, a consecutive part of its k each, and four more add their sums
// in order, apply the activation and store h, while the first are at the next item: their
// streams of steps run on over the block's items.
//
// The shared experts' items come first: their loads are issued before the routes' tables are
// made, which every block does for itself (a launch of its own for them would take longer
// than their two microseconds).  Then the experts with so few tokens that one DMA
// instruction brings their activations, those with up to 16, and those with more.
template <class E, bool MX, int ACT, int NT>
__global__ __launch_bounds__(2 * FT) void few_gu_kernel(FewArgs a) {
  using F = Fmt<E, MX>;
  constexpr int R = ACT == MOE_ACT_SWIGLU ? 2 : 1, NP = gu_tiles(MX, NT);
  using CS = Classes<E, MX, NT, NP>;
  constexpr int RING = gu_ring(NP);
  __shared__ __attribute__((aligned(1024))) char rings[FW][RING];
  __shared__ f32x4_t red[2][FW][R][NP][64];  // (an item's sums, and the next one's)
  __shared__ FewTables tb;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int q4 = lane >> 4;
  const bool streams = wave < FW;
  const int me = blockIdx.x, all = gridDim.x;  // the block takes the items me, me + all, ...
  const int steps = ceil_div(a.d, F::KS);
  const int s_lo = streams ? steps * wave / FW : 0, n = streams ? steps * (wave + 1) / FW - s_lo : 0;

  auto tables = [&]() {
    if (wave == 2 * FW - 1) build_local_map(a.resident, a.E, tb.lmap);
    for (int i = threadIdx.x; i < 256; i += 2 * FT) tb.slot[i] = 0;
    if (a.E <= 64) few_select_all<2 * FW, 4>(a, tb, blockIdx.x == 0);
    else if (a.E <= 128) few_select_all<2 * FW, 8>(a, tb, blockIdx.x == 0);
    else few_select_all<2 * FW, 16>(a, tb, blockIdx.x == 0);
    __syncthreads();
    few_localise(a, tb, blockIdx.x == 0);
    few_active<CS::Few::CT, CS::More::CT>(a, tb);
  };

  // The block's items lo, lo + all .. below hi of a class: (expert, pass, hidden units).
  int buf = 0;
  auto stream = [&](auto cl, bool shared, int first, int lo, int hi, auto&& between) {
    using C = decltype(cl);
    constexpr int N = C::N;
    const int H = shared ? a.Hs : a.H, n_h = H / 16, per = n_h * C::passes(a.T);
    // an item's expert, first hidden unit and columns
    auto expert = [&](int it) {
      return shared ? 0 : __builtin_amdgcn_readfirstlane((int)tb.expert[first + it / per]);
    };
    auto cols = [&](int it, int r) {
      const int my = lane >= a.T ? -1 : shared ? lane : route_to(a, tb, lane, r);
      return Cols<C>(my, C::MOST == 1 ? 0 : it % per / n_h);
    };
    if (!streams) {
      between();
      for (int it = lo; it < hi; it += all) {
        const int r = expert(it), h0 = it % n_h * 16;
        const Cols<C> c = cols(it, r);
        __syncthreads();  // the item's sums are there
#pragma unroll
        for (int m = 0; m < N; ++m) {
          if (wave - FW != m % FW) continue;
          f32x4_t v[R];
#pragma unroll
          for (int i = 0; i < R; ++i) {
            v[i] = red[buf][0][i][m][lane];
#pragma unroll
            for (int q = 1; q < FW; ++q) v[i] += red[buf][q][i][m][lane];
          }
          // hidden units h0 + 4 q4 .. of column l16's token.  h is rounded to E once, the gate in
          // it: the matrix instruction of bf16 weights takes bf16 only, and a second one on the
          // rest (h - bf16(h)) would double the activations, which are half of the second
          // projections' loads already.  y is then off by 2.3e-3 of its norm, where rounding it
          // alone leaves 1.7e-3; moe_layer_fwd rounds h and each route's output.
          if (c.row[m] >= 0) {
            const float gate = shared ? 1.0f : tb.gate[c.row[m]];
            E* out = static_cast<E*>(shared ? a.hs : a.h) + (size_t)c.row[m] * H + h0 + 4 * q4;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float s = gate * silu_f(v[0][i]);
              out[i] = from_f32<E>(R == 2 ? s * v[R - 1][i] : s);
            }
          }
        }
        buf ^= 1;
      }
      return;
    }
    const unsigned line = MX ? (unsigned)a.d / 2 : (unsigned)a.d * sizeof(E), sline = mx_stride(a.d);
    const char* W = static_cast<const char*>(shared ? a.sgu : a.wgu);
    const uint8_t* S = shared ? a.sgu_s : a.wgu_s;
    Stream<E, MX, R, N, 2, C::XP, RING> st(rings[wave & (FW - 1)], a.d);
    using ST = decltype(st);
    st.weights(line, 16);
    if constexpr (MX) st.soff = (unsigned)(min(lane >> 4, R - 1) * H + (lane & 15)) * sline;
    int left = hi > lo ? (hi - lo + all - 1) / all * n : 0;
    int flying = 0, l_slot = 0, l_it = lo, l_s = 0;
    uint64_t w[R], sc = 0;
    const uint64_t x = uniform64(a.x);
    auto issue = [&]() {
      if (left == 0) return;
      if (l_s == 0) {
        const int r = expert(l_it), h0 = l_it % n_h * 16;
        const Cols<C> c = cols(l_it, r);
#pragma unroll
        for (int i = 0; i < N; ++i) st.column(i, c.row[i] >= 0 ? c.t[i] : 0);
#pragma unroll
        for (int i = 0; i < R; ++i) w[i] = uniform64(W + ((size_t)r * R * H + (size_t)i * H + h0) * line);
        if constexpr (MX) sc = uniform64(S + ((size_t)r * R * H + h0) * sline);
      }
      st.issue(l_slot, s_lo + l_s, w, sc, x);
      l_slot = l_slot + 1 == ST::D ? 0 : l_slot + 1;
      if (++l_s == n) {
        l_s = 0;
        l_it += all;
      }
      --left;
      ++flying;
    };
#pragma unroll 1
    for (int i = 0; i < ST::D; ++i) issue();  // (unrolled, its code took longer to fetch than to run)
    between();
    int slot = 0;
    for (int it = lo; it < hi; it += all) {
      f32x4_t acc[R][N];
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int m = 0; m < N; ++m) acc[i][m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      for (int s = 0; s < n; ++s) {
        wait_vm_groups<ST::PER, ST::D - 1>(flying - 1);
        typename ST::Frags f;
        st.read(f, slot, s_lo + s);
        slot = slot + 1 == ST::D ? 0 : slot + 1;
        WAIT_LGKMCNT(0);  // the operands are in registers: their place may be refilled
        --flying;
        issue();
        ST::mma(f, acc);
      }
      // (this buffer's sums of two items ago were read before the last barrier)
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int m = 0; m < N; ++m) red[buf][wave][i][m][lane] = acc[i][m];
      __syncthreads();
      buf ^= 1;
    }
  };

  typedef typename CS::Few Few;
  typedef typename CS::More More;
  typedef typename CS::All All;
  const int n_s = a.Hs / 16 * (a.T <= Few::CT ? 1 : All::passes(a.T)), n_r = a.H / 16;
  // the first of this block's numbers from `from` on
  auto next = [&](int from) {
    const int m = (from - me) % all;
    return from + (m > 0 ? all - m : -m);
  };
  auto nothing = [] {};
  if (a.T <= Few::CT) stream(Few{}, true, 0, me, n_s, tables);
  else stream(All{}, true, 0, me, n_s, tables);
  int from = n_s, first = 0;
  auto routed = [&](auto cl, int experts) {
    const int n_i = experts * n_r * decltype(cl)::passes(a.T);
    stream(cl, false, first, next(from) - from, n_i, nothing);
    from += n_i;
    first += experts;
  };
  routed(Few{}, tb.n_class[0]);
  routed(More{}, tb.n_class[1]);
  if constexpr (16 * NT > More::CT) routed(All{}, tb.n_class[2]);
}

// ------------------------------------------------------------------ second projections
// A block is RB columns of y (rows of W_d; the matrix instruction's other rows are not used)
// and the whole reduction: the shared experts' hidden units, then all active experts', in
// steps of which each wave takes consecutive ones, its stream running on from expert to
// expert.  An expert's sums are added to the wave's own rows of y in LDS, and the waves' rows
// in order at the end.  RB is 16, or 8 where that would leave CUs without a block (bf16, H =
// 1408, us with 16 / 8 / 4 columns: d = 4096, 32 tokens 38 / 48 / 77; 2048, 32 tokens 52 / 42 /
// 66; 2048, one token 15.1 / 14.3 / 23; 1024, 32 tokens 21.0 / 19.6 / 20.5).  Cutting the
// reduction into parts instead, added by the last block to finish, took three times as long
// (the fences write back each XCD's whole L2).
template <class E, bool MX, int NT, int RB>
__global__ __launch_bounds__(DT) void few_down_kernel(FewArgs a) {
  using F = Fmt<E, MX>;
  constexpr int NP = down_tiles(MX, NT);
  using CS = Classes<E, MX, NT, NP>;
  constexpr int WP = RB < 16 ? 1 : 2;
  __shared__ __attribute__((aligned(1024))) char rings[DW][down_ring(NT)];
  __shared__ f32x4_t red[DW][16 * NT][RB / 4];
  __shared__ FewTables tb;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, q4 = lane >> 4;
  for (int i = lane; i < 16 * NT * (RB / 4); i += 64) (&red[wave][0][0])[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  auto tables = [&]() {
    for (int i = threadIdx.x; i < a.T * a.k; i += DT) tb.local[i] = (int16_t)a.w_local[i];
    for (int i = threadIdx.x; i < 256; i += DT) tb.slot[i] = 0;
    __syncthreads();
    few_active<CS::Few::CT, CS::More::CT>(a, tb);
  };

  // The wave's share of the steps of `experts` experts (`passes` over each).
  auto stream = [&](auto cl, bool shared, int first, int experts, auto&& between) {
    using C = decltype(cl);
    constexpr int N = C::N;
    const int H = shared ? a.Hs : a.H, n_h = ceil_div(H, F::KS), passes = C::passes(a.T);
    const int64_t all = (int64_t)experts * passes * n_h;
    const int s_lo = (int)(all * wave / DW), s_hi = (int)(all * (wave + 1) / DW);
    const unsigned line = MX ? (unsigned)H / 2 : (unsigned)H * sizeof(E), sline = mx_stride(H);
    const char* W = static_cast<const char*>(shared ? a.sd : a.wd) + (size_t)blockIdx.x * RB * line;
    const uint8_t* S = (shared ? a.sd_s : a.wd_s) + (size_t)blockIdx.x * RB * sline;
    Stream<E, MX, 1, N, WP, C::XP, down_ring(NT)> st(rings[wave], H);
    using ST = decltype(st);
    st.weights(line, RB);
    if constexpr (MX) st.soff = (unsigned)min(l16, RB - 1) * sline;
    // pass v = expert * passes + pass: its columns
    auto expert = [&](int v) {
      return shared ? 0 : __builtin_amdgcn_readfirstlane((int)tb.expert[first + v / passes]);
    };
    auto cols = [&](int v, int r) {
      const int my = lane >= a.T ? -1 : shared ? lane : route_to(a, tb, lane, r);
      return Cols<C>(my, v % passes);
    };
    // the step to load next: slot of the ring, pass, step in it
    int left = s_hi - s_lo, flying = 0, l_slot = 0, l_v = n_h ? s_lo / n_h : 0, l_s = s_lo - l_v * n_h;
    bool fresh = true;
    uint64_t w = 0, sc = 0;
    const uint64_t x = uniform64(shared ? a.hs : a.h);
    auto issue = [&]() {
      if (left == 0) return;
      if (fresh) {
        fresh = false;
        const int r = expert(l_v);
        const Cols<C> c = cols(l_v, r);
#pragma unroll
        for (int i = 0; i < N; ++i) st.column(i, max(c.row[i], 0));
        w = uniform64(W + (size_t)r * a.d * line);
        if constexpr (MX) sc = uniform64(S + (size_t)r * a.d * sline);
      }
      st.issue(l_slot, l_s, &w, sc, x);
      l_slot = l_slot + 1 == ST::D ? 0 : l_slot + 1;
      if (++l_s == n_h) {
        l_s = 0;
        ++l_v;
        fresh = true;
      }
      --left;
      ++flying;
    };
    int v = l_v, s = l_s, slot = 0, todo = left;
#pragma unroll 1
    for (int i = 0; i < ST::D; ++i) issue();  // (unrolled, its code took longer to fetch than to run)
    between();
    while (todo > 0) {
      f32x4_t acc[1][N];
#pragma unroll
      for (int i = 0; i < N; ++i) acc[0][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      int n = min(todo, n_h - s);
      todo -= n;
      // two steps at a time, so that a wave waits half as often for its operands
      for (; n >= 2; n -= 2, s += 2) {
        wait_vm_groups<ST::PER, ST::D - 2>(flying - 2);
        typename ST::Frags f, g;
        st.read(f, slot, s);
        slot = slot + 1 == ST::D ? 0 : slot + 1;
        st.read(g, slot, s + 1);
        slot = slot + 1 == ST::D ? 0 : slot + 1;
        WAIT_LGKMCNT(0);  // the operands are in registers: their places may be refilled
        flying -= 2;
        issue();
        issue();
        ST::mma(f, acc);
        ST::mma(g, acc);
      }
      if (n) {
        wait_vm_groups<ST::PER, ST::D - 1>(flying - 1);
        typename ST::Frags f;
        st.read(f, slot, s);
        slot = slot + 1 == ST::D ? 0 : slot + 1;
        WAIT_LGKMCNT(0);
        --flying;
        issue();
        ST::mma(f, acc);
      }
      s = 0;
      const Cols<C> c = cols(v, expert(v));
      ++v;
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (c.row[i] >= 0 && 4 * q4 < RB) red[wave][c.t[i]][q4] += acc[0][i];
    }
  };
  typedef typename CS::Few Few;
  typedef typename CS::More More;
  typedef typename CS::All All;
  if (a.T <= Few::CT) stream(Few{}, true, 0, a.Hs ? 1 : 0, tables);
  else stream(All{}, true, 0, a.Hs ? 1 : 0, tables);
  auto nothing = [] {};
  stream(Few{}, false, 0, tb.n_class[0], nothing);
  stream(More{}, false, tb.n_class[0], tb.n_class[1], nothing);
  if constexpr (16 * NT > More::CT)
    stream(All{}, false, tb.n_class[0] + tb.n_class[1], tb.n_class[2], nothing);
  __syncthreads();
  for (int i = threadIdx.x; i < a.T * (RB / 4); i += DT) {
    const int t = i / (RB / 4), c = i % (RB / 4);
    f32x4_t v = red[0][t][c];
#pragma unroll
    for (int q = 1; q < DW; ++q) v += red[q][t][c];
    E* y = static_cast<E*>(a.y) + (size_t)t * a.d + blockIdx.x * RB + 4 * c;
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = from_f32<E>(v[j]);
  }
}

template <class E, bool MX, int ACT, int NT>
void few_launch(const FewArgs& a, hipStream_t s) {
  const int64_t items = std::min<int64_t>(a.E_r, (int64_t)a.T * a.k) * (a.H / 16) + a.Hs / 16;
  const int cus = num_cus(), blocks = (int)std::max<int64_t>(1, std::min<int64_t>(items, cus));
  MOE_TIMED("few_gu", s, few_gu_kernel<E, MX, ACT, NT><<<blocks, 2 * FT, 0, s>>>(a));
#define FEW_DOWN(RB) \
  MOE_TIMED("few_down", s, few_down_kernel<E, MX, NT, RB><<<a.d / RB, DT, 0, s>>>(a))
  if (a.d / 16 >= cus) FEW_DOWN(16);
  else FEW_DOWN(8);
#undef FEW_DOWN
}
}  // namespace

// The launches by type of weights (few_bf16.hip, few_mx.hip, few_f32.hip).
void run_few_bf16(const FewArgs& a, bool swiglu, hipStream_t s);
void run_few_mx(const FewArgs& a, bool swiglu, hipStream_t s);
void run_few_f32(const FewArgs& a, bool swiglu, hipStream_t s);

}  // namespace moe
