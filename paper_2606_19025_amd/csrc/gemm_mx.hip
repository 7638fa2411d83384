// Grouped expert FFN forward in MXFP4: rows and weights in 4-bit floats with a scale per 32
// (mx.h), products on v_mfma_scale_f32_16x16x128_f8f6f4 with fp32 accumulation.
//
//   kind  C                A (row = group token)   B            epilogue
//   GU    [G|U]  N = 2H    x codes [cap, d]        w_gate_up    h = silu(G) U, quantised
//   UP    A      N = H     x codes [cap, d]        w_gate_up    h = silu(A), quantised
//   DOWN  Y      N = d     h codes [cap, H]        w_down       bf16
//
// Persistent blocks over output tiles (ragged in M: laid over the groups from the device-side
// offsets).  A k-step is 256 of k, 128 bytes of a row: a stage of the two-stage LDS ring holds
// the rows' code pieces and 8 bytes of scales each, all by DMA through buffer resources
// (offsets past the range read zeros: what a cut last k-step lacks).  A 16-byte chunk c of
// row r sits at chunk c ^ ((r >> 1) & 7), so that operand reads are free of bank conflicts.
// A 4-bit operand of this instruction is as many bytes as a bf16 one of the 16x16x32
// form and as long a pass of the matrix unit: per byte brought to LDS and read from it the
// kernel does four times the arithmetic of the bf16 GEMM.
//
// A k-step is 2 NJ chunks of MI products; a chunk's columns are read four chunks ahead.  Four
// chunks before its end all of the stage has been read: the wave waits for the next
// stage's DMA, takes the barrier (this stage is free, the next is whole) and refills it.
// A tile's first two stages are issued before the previous tile's epilogue.
//
// Measured (65536 rows in 32 groups, d = 4096, H = 2048): first projection 658 us, second 400:
// 3.3 and 2.7 PFLOP/s, by the clock that power leaves (1.76 GHz; calls apart 580 and 375).  Over
// both the matrix units are busy 41 % of the time, the LDS pipe about as much (operands and
// scales 27, conflicts 3, the DMA's writes some 11): what is left are the waits at each k-step's
// barrier and the epilogues, which have no products beside them.
#include "gemm.h"
#include "kernels.h"
#include "mx.h"
#include "timing.h"

namespace moe {
namespace {

enum MxKind { MX_GU = 0, MX_UP = 1, MX_DOWN = 2 };

typedef int i32x8_v __attribute__((ext_vector_type(8)));

struct MxGemmArgs {
  GemmArgs g;              // offsets, n_groups, cap (for the group table)
  const uint8_t *a, *as;   // codes and scales of the rows [cap, K]
  const uint8_t *b, *bs;   // and of the weights [groups, N, K]
  uint8_t *h, *hs;         // GU, UP: codes and scales of h [cap, H]
  bf16_t* y;               // DOWN: [cap, N]
  int K, N, H;
};

// An offset past every operand; the range check holds with a step's offset added too.
constexpr unsigned kPast = 0xFFFFFFF0u;

DEVI u32x4_t mx_rsrc(const void* base, size_t bytes) {
  const uint64_t b = (uint64_t)(uintptr_t)base;
  u32x4_t r;
  r[0] = __builtin_amdgcn_readfirstlane((unsigned)b);
  r[1] = __builtin_amdgcn_readfirstlane((unsigned)(b >> 32) & 0xFFFFu);
  r[2] = __builtin_amdgcn_readfirstlane((unsigned)bytes);
  r[3] = 0x00020000u;
  return r;
}
// 16 bytes per lane at byte offset off + soff (soff uniform) to LDS at lds + 16 lane.  The asm sets m0 and
// leaves the one wait state an LDS DMA needs after it.
DEVI void mx_dma16(u32x4_t rsrc, unsigned off, unsigned soff, unsigned lds) {
  asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds" ::"v"(off), "s"(rsrc),
               "s"(soff), "s"(lds)
               : "m0", "memory");
}

// silu by the hardware's exp2 and reciprocal: for g >= -87.3 off by a few 2^-24 and 1.5 |g| 2^-24
// of itself (the rounding of g log2 e); below, where the exponential or its reciprocal leaves fp32's
// normal numbers, by up to all of it, at most 1.03e-36 (from -88.8 on it is 0).  expf and a division
// made the epilogue a quarter of a tile's time.
DEVI float silu_hw(float g) {
  return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896341f * g));
}

// A block's tile: WR x WC waves of MI x NJ MFMA tiles.
template <int MI_, int NJ_, int WR_, int WC_>
struct MxTile {
  static constexpr int MI = MI_, NJ = NJ_, WR = WR_, WC = WC_, NW = WR * WC, NT = 64 * NW;
  static constexpr int BM = 16 * MI * WR, BN = 16 * NJ * WC;
  static constexpr int PA = BM / (8 * NW), PB = BN / (8 * NW);  // 8-row DMA pieces per wave
  static constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128, STAGE = A_BYTES + B_BYTES;
  static constexpr int SP = (BM + BN) / 64, S_STAGE = NW * 1024;     // 64-row scale pieces
  static constexpr int S_AT = 2 * STAGE, E_AT = S_AT + 2 * S_STAGE;
  static constexpr int EPI = 1024;  // a wave's staging: 8 rows of 64 bf16
  static constexpr int LDS = E_AT + NW * EPI;
  static_assert(SP <= NW && BM % 64 == 0 && BN % 64 == 0, "a scale piece per wave at most");
};

template <int KIND, class T>
__global__ __launch_bounds__(T::NT) void mx_gemm_kernel(MxGemmArgs p) {
  constexpr int MI = T::MI, NJ = T::NJ, NW = T::NW;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  __shared__ GroupTable gt;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, q4 = lane >> 4;
  const int wr = wave / T::WC, wc = wave % T::WC;
  if (wave == 0) build_group_table<T::BM>(p.g, gt, 0);
  __syncthreads();
  const int ng = p.g.n_groups;
  const int n_n = (p.N + T::BN - 1) / T::BN, tiles = gt.p[ng] * n_n;
  const int steps = (p.K + 255) / 256;
  const unsigned line = p.K / 2, sline = mx_stride(p.K);
  const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(lds_void_t*)lds);
  const size_t b_rows = (size_t)ng * p.N;
  const u32x4_t ra = mx_rsrc(p.a, (size_t)p.g.cap * line), rb = mx_rsrc(p.b, b_rows * line);
  const u32x4_t rs = wave * 64 < T::BM ? mx_rsrc(p.as, (size_t)p.g.cap * sline) : mx_rsrc(p.bs, b_rows * sline);

  // Tiles are dealt to the XCDs (blocks are placed on them round-robin) in equal consecutive
  // shares; within a group they run in bands of 4 m-tiles, so that the tiles an XCD runs at
  // a time share rows and weights in its L2.
  const int per_xcd = gridDim.x / 8, xcd = blockIdx.x % 8;
  const int t_end = (int)((int64_t)tiles * (xcd + 1) / 8);
  int tile = (int)((int64_t)tiles * xcd / 8) + blockIdx.x / 8;

  struct Where { int g, row0, row1, n0; };  // rows [row0, row1) of group g, tile column n0
  auto decode = [&](int t) {
    int g = 0;
    for (int g0 = 0; g0 < ng; g0 += 64) {
      const uint64_t m = __ballot(g0 + lane < ng && gt.p[min(g0 + lane, ng - 1) + 1] * n_n > t);
      if (m) {
        g = g0 + __ffsll((unsigned long long)m) - 1;
        break;
      }
    }
    g = __builtin_amdgcn_readfirstlane(g);
    const int m_g = gt.p[g + 1] - gt.p[g], local = t - gt.p[g] * n_n;
    const int band = local / (4 * n_n), rem = local - band * 4 * n_n, high = min(4, m_g - band * 4);
    Where w;
    w.g = g;
    w.n0 = rem / high;
    w.row0 = gt.b[g] + (band * 4 + rem % high) * T::BM;
    w.row1 = min(gt.b[g + 1], w.row0 + T::BM);
    return w;
  };
  // row of the weights at column c of tile column n0 (clamped past the last: not stored)
  auto b_row = [&](int n0, int c) {
    if constexpr (KIND == MX_GU) {  // gate and up in turn, 32 hidden units each
      const int q = c >> 5, hid = min(n0 * (T::BN / 2) + (q >> 1) * 32 + (c & 31), p.H - 1);
      return (q & 1) * p.H + hid;
    } else {
      return min(n0 * T::BN + c, p.N - 1);
    }
  };

  // Lane offsets of the tile at hand.  A wave's pieces are 8 NW rows apart, a multiple of 16:
  // the lane's chunk of its row is the same in all of them.
  static_assert(NW % 2 == 0, "pieces 16 rows apart");
  unsigned oa[T::PA], ob[T::PB], os;
  const int chunk = (lane & 7) ^ (((wave * 8 + (lane >> 3)) >> 1) & 7);
  // (its lane index passes through an asm: kept from tile to tile, parts of the offsets went
  // through scratch memory, and each reload waited for the loads issued before it.  The large
  // tiles still spill 3 to 8 registers, 16 to 36 bytes a lane)
  auto aim = [&](const Where& w) {
    int al = lane;
    asm volatile("" : "+v"(al));
#pragma unroll
    for (int i = 0; i < T::PA; ++i) {
      const int r = (i * NW + wave) * 8 + (al >> 3);
      oa[i] = (unsigned)min(w.row0 + r, w.row1 - 1) * line + ((al & 7) ^ (((wave * 8 + (al >> 3)) >> 1) & 7)) * 16;
    }
    const unsigned bg = (unsigned)w.g * (unsigned)p.N;
#pragma unroll
    for (int i = 0; i < T::PB; ++i) {
      const int r = (i * NW + wave) * 8 + (al >> 3);
      ob[i] = (bg + (unsigned)b_row(w.n0, r)) * line + ((al & 7) ^ (((wave * 8 + (al >> 3)) >> 1) & 7)) * 16;
    }
    // scales: 64 rows of A, then of B, by wave
    const int r = wave * 64 + al;
    os = wave >= T::SP ? kPast : (r < T::BM ? (unsigned)min(w.row0 + r, w.row1 - 1) : bg + (unsigned)b_row(w.n0, r - T::BM)) * sline;
  };
  // Part q of 4 of a k-step's loads; even k-steps bring the scales of two, 16 bytes of a row
  // (8 at a time, their requests to the L2 were as many as the codes').
  auto issue_part = [&](int kt, auto even, int q) {
    const unsigned at = lds0 + (kt & 1) * T::STAGE;
    // the chunks past a cut last k-step read zeros
    const bool in = chunk * 32 < p.K - kt * 256;
#pragma unroll
    for (int i = 0; i < T::PA; ++i)
      if (i % 4 == q) mx_dma16(ra, in ? oa[i] : kPast, kt * 128, at + (i * NW + wave) * 1024);
#pragma unroll
    for (int i = 0; i < T::PB; ++i)
      if (i % 4 == q) mx_dma16(rb, in ? ob[i] : kPast, kt * 128, at + T::A_BYTES + (i * NW + wave) * 1024);
    if (decltype(even)::value && q == 3)
      mx_dma16(rs, os, kt * 8, lds0 + T::S_AT + (kt >> 1 & 1) * T::S_STAGE + wave * 1024);
  };
  auto issue_first = [&]() {
#pragma unroll
    for (int q = 0; q < 4; ++q) issue_part(0, std::true_type{}, q);
    if (steps > 1)
#pragma unroll
      for (int q = 0; q < 4; ++q) issue_part(1, std::false_type{}, q);
  };

  // Operands: the wave's rows of one k128 half, and the columns of one chunk (a half's j).
  // Scales: the words of both halves, read once a k-step, of which a lane's own bytes are
  // packed where they are first used (sooner would wait for the read); the instruction
  // picks the half's byte.
  struct Rows { u32x4_t v[MI]; };
  u32x2_t raw_a[MI], raw_b[4];
  unsigned sa[MI], sb[NJ];
  // a tile's rows are 16 apart: its place in a stage is the first one's plus 2048 bytes each
  // (the other half's chunk is 64 bytes further or back), 256 bytes of scales
  const unsigned place = l16 * 128 + ((q4 ^ ((l16 >> 1) & 7)) << 4), pick = q4 | (4 + q4) << 8;
  const unsigned rows_at = wr * MI * 2048, cols_at = T::A_BYTES + wc * NJ * 2048;
  const unsigned rs_at = T::S_AT + wr * MI * 256 + l16 * 16, cs_at = T::S_AT + T::BM * 16 + wc * NJ * 256 + l16 * 16;
  auto scales = [&](int kt) { return lds + (kt >> 1 & 1) * T::S_STAGE + (kt & 1) * 8; };
  auto pack = [&](u32x2_t w) { return __builtin_amdgcn_perm(w[1], w[0], pick); };
  auto read_rows = [&](Rows& f, int kt, int half) {
    const char* v = lds + (kt & 1) * T::STAGE + rows_at + (place ^ (half * 64));
#pragma unroll
    for (int i = 0; i < MI; ++i) f.v[i] = *reinterpret_cast<const u32x4_t*>(v + i * 2048);
  };
  auto read_row_scales = [&](int kt) {
#pragma unroll
    for (int i = 0; i < MI; ++i) raw_a[i] = *reinterpret_cast<const u32x2_t*>(scales(kt) + rs_at + i * 256);
  };
  auto read_col = [&](u32x4_t& f, int kt, int half, int j) {
    f = *reinterpret_cast<const u32x4_t*>(lds + (kt & 1) * T::STAGE + cols_at + (place ^ (half * 64)) + j * 2048);
    if (half == 0) raw_b[j % 4] = *reinterpret_cast<const u32x2_t*>(scales(kt) + cs_at + j * 256);
  };
  f32x4_t acc[MI][NJ];
  auto wide = [](u32x4_t v) {
    const i32x8_v r = {(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
    return r;
  };
  // the weights are the first operand: a lane holds four consecutive columns of one row
  auto mma = [&](const Rows& a, u32x4_t b, auto half, int j) {
    constexpr int HALF = decltype(half)::value;
#pragma unroll
    for (int i = 0; i < MI; ++i)
      acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(b), wide(a.v[i]), acc[i][j], 4, 4, HALF,
                                                                   (int)sb[j], HALF, (int)sa[i]);
  };

  if (tile >= t_end) return;
  Where w = decode(tile);
  aim(w);
  issue_first();
  // the second word of a cut last k-step may be past the end of its row
  const unsigned past = p.K - (steps - 1) * 256 > 128 ? ~0u : 0xFFu;
  for (;;) {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    WAIT_VMCNT(0);
    __syncthreads();  // the first stages are whole
    // 2 NJ chunks to a k-step, the columns of four of them in registers
    constexpr int C = 2 * NJ;
    Rows a0, a1;
    u32x4_t b[4];
    read_rows(a0, 0, 0);
    read_row_scales(0);
#pragma unroll
    for (int c = 0; c < 4; ++c) read_col(b[c], 0, 0, c);
    // (no branch inside a k-step: the compiler would move its products past it)
    auto step = [&](auto refill, auto next, auto even, int kt) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        if (c == C - 4) {
          WAIT_LGKMCNT(0);
          WAIT_VMCNT(0);
          __syncthreads();  // this stage has been read, the next one is whole
          if constexpr (decltype(next)::value) {
            read_rows(a0, kt + 1, 0);
            read_row_scales(kt + 1);
          }
        }
        const unsigned mask = decltype(next)::value ? ~0u : past;
        if (c == 0) {
#pragma unroll
          for (int i = 0; i < MI; ++i) sa[i] = pack(raw_a[i]) & mask;
        }
        if (c == 1) read_rows(a1, kt, 1);
        if (c < NJ) {
          sb[c] = pack(raw_b[c % 4]) & mask;
          mma(a0, b[c % 4], std::integral_constant<int, 0>{}, c);
        } else {
          mma(a1, b[c % 4], std::integral_constant<int, 1>{}, c - NJ);
        }
        if (c + 4 < C) read_col(b[c % 4], kt, (c + 4) / NJ, (c + 4) % NJ);
        else if constexpr (decltype(next)::value) read_col(b[c % 4], kt + 1, 0, c + 4 - C);
        if constexpr (decltype(refill)::value)
          if (c >= C - 4) issue_part(kt + 2, even, c - (C - 4));
        __builtin_amdgcn_sched_barrier(0);  // (reads moved further ahead cost registers)
      }
    };
    typedef std::true_type Yes;
    typedef std::false_type No;
    int kt = 0;
    while (kt + 2 < steps) {
      step(Yes{}, Yes{}, Yes{}, kt++);
      if (kt + 2 < steps) step(Yes{}, Yes{}, No{}, kt++);
    }
    if (kt + 1 < steps) step(No{}, Yes{}, No{}, kt++);
    step(No{}, No{}, No{}, kt);
    // (the last products stay here: moved past the branch below, their operands went through
    // scratch memory and waited for the next tile's loads; 65536 rows, first projection 790
    // us and then 680, second 465 and 398)
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) asm volatile("" : "+v"(acc[i][j]));
    // the next tile's first stages, while this one's results are stored
    const Where done = w;
    const bool more = tile + per_xcd < t_end;
    if (more) {
      tile += per_xcd;
      w = decode(tile);
      aim(w);
      issue_first();
    }
    const int m0 = done.row0 + wr * MI * 16;  // this wave's first row
    // (the epilogue's lane index passes through an asm, so that its addresses are computed
    // here and not kept in registers through the main loop)
    int el = lane;
    asm volatile("" : "+v"(el));
    const int l16 = el & 15, q4 = el >> 4;
    if constexpr (KIND == MX_DOWN) {
      // 8 rows of 64 columns at a time through the wave's staging, so that a store covers
      // 128 bytes of a row; 16-byte chunk c of row r at chunk c ^ r
      char* stage = lds + T::E_AT + wave * T::EPI;
      const int c0 = done.n0 * T::BN + wc * NJ * 16;
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int jh = 0; jh < NJ; jh += 4)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            if (l16 >> 3 == u) {
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const f32x4_t v = acc[i][jh + j];
                const bf16x4_t o = {(bf16_t)v[0], (bf16_t)v[1], (bf16_t)v[2], (bf16_t)v[3]};
                const int r = l16 & 7;
                *reinterpret_cast<bf16x4_t*>(stage + r * 128 + (((2 * j + (q4 >> 1)) ^ r) << 4) + (q4 & 1) * 8) = o;
              }
            }
            const int r = el >> 3, c = el & 7;
            const u32x4_t v = *reinterpret_cast<const u32x4_t*>(stage + r * 128 + ((c ^ r) << 4));
            const int row = m0 + i * 16 + u * 8 + r, col = c0 + jh * 16 + c * 8;
            // (past the caches: y is not read again here)
            if (row < done.row1 && col < p.N)
              __builtin_nontemporal_store(v, reinterpret_cast<u32x4_t*>(p.y + (size_t)row * p.N + col));
          }
    } else {
      // h of 32 hidden units (a block) of row l16: 8 values in each of the lanes l16 + 16 q
      constexpr int HB = KIND == MX_GU ? NJ / 4 : NJ / 2;
      const int hb0 = (done.n0 * T::WC + wc) * HB;  // the wave's first block
      const unsigned hline = p.H / 2, hsline = mx_stride(p.H);
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int b = 0; b < HB; ++b) {
          float v[8];
          unsigned top = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int j = (e >> 2) + (KIND == MX_GU ? 4 * b : 2 * b);
            const float g = acc[i][j][e & 3];
            v[e] = silu_hw(g);
            if constexpr (KIND == MX_GU) v[e] *= acc[i][j + 2][e & 3];
            top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);
          }
          top = max(top, (unsigned)__shfl_xor((int)top, 16, 64));
          top = max(top, (unsigned)__shfl_xor((int)top, 32, 64));
          const unsigned s = mx_scale_code(top);
          const unsigned c = mx_codes8(v, s);  // columns 4 q .. and 16 + 4 q ..
          // lane q's word of the block's sixteen bytes: columns 8 q .. 8 q + 7
          const unsigned lo = (unsigned)__shfl((int)c, l16 + 32 * (q4 & 1), 64);
          const unsigned hi = (unsigned)__shfl((int)c, l16 + 32 * (q4 & 1) + 16, 64);
          const unsigned word = q4 < 2 ? (lo & 0xffffu) | hi << 16 : lo >> 16 | (hi & 0xffff0000u);
          const int row = m0 + i * 16 + l16, blk = hb0 + b;
          if (row < done.row1 && blk * MX_BLOCK < p.H) {
            *reinterpret_cast<unsigned*>(p.h + (size_t)row * hline + blk * 16 + q4 * 4) = word;
            if (q4 == 0) {
              uint8_t* out = p.hs + (size_t)row * hsline;
              out[blk] = (uint8_t)s;
              if ((blk + 1) * MX_BLOCK == p.H)  // the bytes past the last block are zero
                for (unsigned z = blk + 1; z < hsline; ++z) out[z] = 0;
            }
          }
        }
    }
    if (!more) break;
  }
}

typedef MxTile<4, 8, 4, 2> MxLarge;  // 256 x 256
typedef MxTile<2, 4, 2, 2> MxSmall;  // 64 x 128

template <int KIND, class T>
hipError_t mx_run(const MxGemmArgs& a, const char* name, hipStream_t s) {
  static_assert(T::LDS + sizeof(GroupTable) <= 160 * 1024, "LDS");
  const int blocks = num_cus() / 8 * 8 * (T::LDS * 2 <= 150 * 1024 ? 2 : 1);
  MOE_TIMED(name, s, mx_gemm_kernel<KIND, T><<<blocks, T::NT, T::LDS, s>>>(a));
  return hipGetLastError();
}

// Large tiles read each operand fewer times, small ones fill the CUs sooner (two blocks on
// each) and pad small groups less.  Large where the rows, all there and spread evenly, give every
// CU a tile that is more than half full.
// Measured (us, large / small, and the large tiles; rows, groups, d, H):
//                            first projection   second
//   128, 128, 2048, 1408      140 /  74  704      70 /  47  512
//   256, 256, 1024, 1408      169 /  78 1419      72 /  48  516
//   2048, 16, 2048, 1408       24 /  20  176      18 /  13  128
//   4096,  8, 1024, 2816       32 /  33  440      25 /  16   80
//   8192,  4, 1024, 2816       45 /  59  748      25 /  25  136
//   8192,  8, 4096, 1024       41 /  61  288      33 /  38  576
//   8192, 16, 2048, 1408       44 /  50  440      23 /  32  320
//   16384, 8, 1024, 2816       85 / 113 1496      31 /  46  272
//   65536, 32, 4096, 2048     595 / 974 4352     380 / 529 4352
// and by rows of a group (the tiles of small groups are mostly padding):
//          64 groups, 2048, 1408     32 groups, 4096, 2048     256 groups, 1024, 704
//   64       75 /  51   41 /  32       88 /  67   47 /  35       98 /  54   56 /  38
//   96       77 /  69   43 /  44       91 /  92   51 /  50       99 /  76   59 /  54
//  128       77 /  71   44 /  48       94 /  98   52 /  54      101 /  78   63 /  60
//  160       79 /  88   47 /  59       94 / 114   54 /  65      102 /  99   68 /  72
//  192       80 /  89   49 /  61       96 / 118   56 /  68      105 / 102   73 /  77
//  256       82 / 118   54 /  83       99 / 163   60 /  94      108 / 138   80 / 108
// The rows that are there are known on the device only.  With a quarter of cap's (6144 in 16
// groups, 2048, 1408: 24 / 19, 18 / 12; 16384 in 8, 1024, 2816: 31 / 31, 25 / 15; 16384 in 16,
// 2048, 1408: 25 / 29, 19 / 18) the choice for all of them is up to half again slower.
template <int KIND>
hipError_t mx_launch(const MxGemmArgs& a, const char* name, hipStream_t s) {
  const int64_t tiles =
      (int64_t)(a.g.cap / MxLarge::BM + (a.g.n_groups + 1) / 2) * ceil_div(a.N, MxLarge::BN);
  const bool large = tiles >= num_cus() && a.g.cap > MxLarge::BM / 2 * a.g.n_groups;
  return large ? mx_run<KIND, MxLarge>(a, name, s) : mx_run<KIND, MxSmall>(a, name, s);
}

}  // namespace

size_t mx_ffn_ws_bytes(int cap, int H) {
  const size_t codes = ((size_t)cap * H / 2 + 255) & ~(size_t)255;
  return codes + (size_t)cap * mx_stride(H);
}

hipError_t launch_mx_ffn(const moe_mxfp4_ffn* f, hipStream_t s) {
  if (f->cap == 0 || f->n_groups == 0) return hipSuccess;
  MxGemmArgs a{};
  a.g.offsets = f->offsets;
  a.g.n_groups = f->n_groups;
  a.g.cap = f->cap;
  a.H = f->H;
  a.h = static_cast<uint8_t*>(f->ws);
  a.hs = a.h + (((size_t)f->cap * f->H / 2 + 255) & ~(size_t)255);
  a.a = f->x; a.as = f->x_scales; a.b = f->w_gate_up; a.bs = f->w_gate_up_scales;
  a.K = f->d;
  const bool swiglu = f->activation == MOE_ACT_SWIGLU;
  a.N = swiglu ? 2 * f->H : f->H;
  hipError_t e = swiglu ? mx_launch<MX_GU>(a, "mx_gemm_gu", s) : mx_launch<MX_UP>(a, "mx_gemm_up", s);
  if (e != hipSuccess) return e;
  a.a = a.h; a.as = a.hs; a.b = f->w_down; a.bs = f->w_down_scales;
  a.y = static_cast<bf16_t*>(f->y);
  a.K = f->H;
  a.N = f->d;
  return mx_launch<MX_DOWN>(a, "mx_gemm_down", s);
}

}  // namespace moe
