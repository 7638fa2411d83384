// The norms and the residual sum around a block of a Peri-LN transformer
// (x + LN(F(LN(x))), App. B): the block's output norm, its gate and residual scale,
// the sum, and the input norm of the next block in one pass over the rows.
//
//   n  = post ? (f - mu_f) r_f w_post + b_post : f
//   x' = x + a g n            (g: 1, one per channel or one per token), rounded to its type
//   u  = (x' - mu_x) r_x w_pre + b_pre          (of the rounded x', which the backward reads)
//   backward, with xh, fh the normalised rows and LN'(q, h, r) = r (q - mean q - h mean(q h)):
//     G  = dres + LN'(du w_pre, xh, r_x) = dx;   dn = a g G;   df = LN'(dn w_post, fh, r_f)
//     dw_pre = sum_t du xh,  db_pre = sum_t du,  dw_post = sum_t dn fh,  db_post = sum_t dn
//     dg[c] = a sum_t G n,   dg[t] = a sum_c G n
//
// Bound by HBM: forward two arrays read and two written, backward four and two (as single
// operators seven and ten).  Rows stay in registers as fp32, as in norm.hip.  The column sums
// of the backward need two rows of products more than a norm's: with a gate per channel
// dw_post, db_post and dg are g S3, g S4 and w S3 + b S4 of S3 = sum a G fh, S4 = sum a G, so
// that four sums do for five gradients; a block keeps them in registers, stores one partial
// row of 4 d and a second launch adds the partials in a fixed order.
//
// Measured (bf16, a gate per channel; second launch included): 8192 x 2048 forward 29 us, backward 48; 16384 x
// 4096 109 and 155 us (4.9 and 5.2 TB/s); 8192 x 1024 14 and 31; fp32 8192 x 2048 53 and 80 (5.1, 5.0 TB/s).
#include "common.h"
#include "kernels.h"
#include "norm_rows.h"
#include "timing.h"

namespace moe {
namespace {

constexpr int kSums = 4;  // column sums of the backward

struct BlockArgs {
  moe_block_norm p;
  float* part;  // backward: [blocks][4][d]
  float inv_d;
};

// v + the value of the lane N back in its row of 16, in a ring.
template <int N>
DEVI float add_ror(float v) {
  return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + N, 0xf,
                                                                   0xf, false));
}

// Sums of N values over the W waves of a row, in all their lanes, as row_sums; across a wave by
// moves between lanes (within rows of 16, then swaps of rows and of halves), which take no LDS.
DEVI float lane_sum(float v) {
  v = add_ror<1>(add_ror<2>(add_ror<4>(add_ror<8>(v))));
  const unsigned u = __builtin_bit_cast(unsigned, v);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  v = __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
  const unsigned h = __builtin_bit_cast(unsigned, v);
  const auto q = __builtin_amdgcn_permlane32_swap(h, h, false, false);
  return __builtin_bit_cast(float, (unsigned)q[0]) + __builtin_bit_cast(float, (unsigned)q[1]);
}
template <int W, int N>
DEVI void all_sums(float (&v)[N], float (*buf)[W], int& flip) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = lane_sum(v[i]);
  if constexpr (W > 1) {
    float (*p)[W] = buf + flip * N;
    flip ^= 1;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) p[i][(threadIdx.x >> 6) % W] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float u = p[i][threadIdx.x % W];  // (a lane's neighbours hold the other waves')
      if (W > 8) u = add_ror<8>(u);
      if (W > 4) u = add_ror<4>(u);
      if (W > 2) u = add_ror<2>(u);
      v[i] = add_ror<1>(u);
    }
  }
}

// mean and 1 / deviation of v (zeros past the row's end), which becomes v - mean
template <class R, int W, int NV>
DEVI void center(const BlockArgs& a, float (&v)[NV][R::VE], float (*buf)[W], int& flip, float& mu,
                 float& r) {
  float s[1] = {0.f};
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < R::VE; ++j) s[0] += v[i][j];
  all_sums<W>(s, buf, flip);
  mu = s[0] * a.inv_d;
  s[0] = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (R::col(i) < a.p.d)
#pragma unroll
      for (int j = 0; j < R::VE; ++j) {
        v[i][j] -= mu;
        s[0] += v[i][j] * v[i][j];
      }
  all_sums<W>(s, buf, flip);
  r = 1.0f / sqrtf(s[0] * a.inv_d + a.p.eps);
}

// The lane's pieces of a row of `bytes` bytes at base -> LDS at dst + 1024 i + 16 lane (dst of the
// wave's own, base wave-uniform); zeros past the row's end.  The asm sets m0 and leaves the one
// wait state that an LDS DMA needs after it.
template <int W, int NV>
DEVI void dma_row(const void* base, int bytes, int wave, char* dst) {
  const uint64_t b = (uint64_t)(uintptr_t)base;
  const u32x4_t r = {(unsigned)__builtin_amdgcn_readfirstlane((unsigned)b),
                     (unsigned)__builtin_amdgcn_readfirstlane((unsigned)(b >> 32) & 0xFFFFu),
                     (unsigned)__builtin_amdgcn_readfirstlane((unsigned)bytes), 0x00020000u};
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const unsigned off = (unsigned)(((i * W + wave) * 64 + (int)(threadIdx.x & 63)) * 16);
    const unsigned m0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(lds_void_t*)(dst + i * 1024));
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(off), "s"(r), "s"(m0)
                 : "m0", "memory");
  }
}

// Waves of a block: kBlockWaves / W groups of W waves take a row each.
constexpr int kBlockWaves = 8;
constexpr int row_block_waves(int W) { return W > kBlockWaves ? W : kBlockWaves; }

// Rows of up to 8 values a lane.  A block's groups of W waves take rows in turn, in step with each other; the
// next rows' f and x come by DMA into LDS while these are worked on, each wave reading what its own lanes
// asked for, so that no barrier is needed for them.  Weights stay in registers.  Three blocks of eight waves
// a CU (two or four: 4096 x 2048 15.4 or 15.5 us and not 14.4, 20000 x 2056 91 or 87 and not 80; 8192 x 2048
// 28.9 or 31 and 29.5), one of sixteen (4096 x 8192 56 us, with two 60).  64 registers for four spill: 60 us
// at 8192 x 2048.  Instead of this, a wave or a block for each row: 8192 x 2048 34 us, 16384 x 4096 118 (now
// 109), 65536 x 256 46 (34); better at 9000 x 1032 alone, 21 (23), where half the lanes hold nothing.
// PRE, POST: the norms that there are.
template <class E, int W, int NV, bool PRE, bool POST>
__global__ __launch_bounds__(64 * row_block_waves(W), 4) void block_norm_fwd_kernel(BlockArgs a) {
  using R = Row<E, W, NV>;
  constexpr int VE = R::VE, BW = row_block_waves(W), GROUPS = BW / W, WAVE = 2 * NV * 1024;
  __shared__ __attribute__((aligned(16))) char ring[2][BW][WAVE];
  __shared__ float buf[GROUPS][2][W];
  const moe_block_norm& p = a.p;
  const bool channel = p.gate_kind == MOE_BLOCK_GATE_CHANNEL;
  const bool token = p.gate_kind == MOE_BLOCK_GATE_TOKEN;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int group = wave / W, wr = wave % W;
  const int step = gridDim.x * GROUPS;
  float wpre[NV][VE], bpre[NV][VE], wpost[NV][VE], bpost[NV][VE], g[NV][VE];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      wpre[i][j] = bpre[i][j] = wpost[i][j] = bpost[i][j] = 0.f;
      g[i][j] = 1.f;
    }
    if (R::col(i) < p.d) {
      if (PRE) R::load_f32(p.pre_weight, R::col(i), wpre[i]);
      if (PRE && p.pre_bias) R::load_f32(p.pre_bias, R::col(i), bpre[i]);
      if (POST) R::load_f32(p.post_weight, R::col(i), wpost[i]);
      if (POST && p.post_bias) R::load_f32(p.post_bias, R::col(i), bpost[i]);
      if (channel) R::load_f32(p.gate, R::col(i), g[i]);
    }
  }
  const int bytes = p.d * (int)sizeof(E);
  float ng = 1.f;
  auto fetch = [&](int t, char* dst) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (what was there has been read)
    const int n = t < p.T ? bytes : 0;
    const size_t at = t < p.T ? (size_t)t * p.d : 0;
    dma_row<W, NV>(static_cast<const E*>(p.f) + at, n, wr, dst);
    dma_row<W, NV>(static_cast<const E*>(p.x) + at, n, wr, dst + NV * 1024);
    if (token) ng = p.gate[min(t, p.T - 1)];
  };
  auto read = [&](const char* src, int k, int i, float* out) {
    R::unpack(*reinterpret_cast<const u32x4_t*>(src + (k * NV + i) * 1024 + lane * 16), out);
  };
  int flip = 0, cur = 0;
  float (*sums)[W] = buf[group];
  const int first = blockIdx.x * GROUPS;
  if (first < p.T) fetch(first + group, ring[0][wave]);
  for (int t0 = first; t0 < p.T; t0 += step) {  // (as often in all waves)
    const int t = t0 + group;
    const bool there = t < p.T;
    // These rows have landed (the last rows' stores too: the loads that the compiler tracks, of a token's gate,
    // make it wait for all in any case, so no count of what is newer than the DMA would let them pass)
    asm volatile("s_waitcnt vmcnt(0)" : "+v"(ng)::"memory");
    const float ag = p.scale * ng;
    const char* src = ring[cur][wave];
    cur ^= 1;
    if (t0 + step < p.T) fetch(t + step, ring[cur][wave]);
    float n[NV][VE], mu, r = 1.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) read(src, 0, i, n[i]);
    if constexpr (POST) {
      center<R, W, NV>(a, n, sums, flip, mu, r);
      if (there && wr == 0 && lane == 0) {
        p.post_mean[t] = mu;
        p.post_rstd[t] = r;
      }
    }
    E* xo = static_cast<E*>(p.x_out) + (size_t)t * p.d;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float x[VE];
      read(src, 1, i, x);
      const bool in = R::col(i) < p.d;
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        // (past the row's end x' is a zero)
        const float v = POST ? n[i][j] * r * wpost[i][j] + bpost[i][j] : n[i][j];
        n[i][j] = in ? (float)from_f32<E>(x[j] + ag * (v * g[i][j])) : 0.f;
      }
      if (there && in) store16_f32(xo + R::col(i), n[i]);
    }
    if constexpr (PRE) {
      center<R, W, NV>(a, n, sums, flip, mu, r);
      if (there && wr == 0 && lane == 0) {
        p.pre_mean[t] = mu;
        p.pre_rstd[t] = r;
      }
      E* u = static_cast<E*>(p.u) + (size_t)t * p.d;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int j = 0; j < VE; ++j) n[i][j] = n[i][j] * r * wpre[i][j] + bpre[i][j];
        if (there && R::col(i) < p.d) store16_f32(u + R::col(i), n[i]);
      }
    }
  }
}

// Wide rows, 16 values a lane of a block of sixteen waves for each row.
template <class E>
__global__ __launch_bounds__(1024) void block_norm_fwd_wide_kernel(BlockArgs a) {
  constexpr int W = 16, VE = Vec16<E>::N, NV = 16 / VE;
  using R = Row<E, W, NV>;
  __shared__ float buf[2][W];
  const moe_block_norm& p = a.p;
  const int t = blockIdx.x;
  const bool first = threadIdx.x == 0;
  u32x4_t rf[NV], rx[NV];
  R::load(p.f, t, p.d, rf);
  R::load(p.x, t, p.d, rx);
  int flip = 0;
  float mu, r = 1.f;
  float n[NV][VE];
#pragma unroll
  for (int i = 0; i < NV; ++i) R::unpack(rf[i], n[i]);
  if (p.post_weight) {
    center<R, W, NV>(a, n, buf, flip, mu, r);
    if (first) {
      p.post_mean[t] = mu;
      p.post_rstd[t] = r;
    }
  }
  const float ag = p.gate && p.gate_kind == MOE_BLOCK_GATE_TOKEN ? p.scale * p.gate[t] : p.scale;
  E* xo = static_cast<E*>(p.x_out) + (size_t)t * p.d;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = R::col(i);
    float x[VE];
    R::unpack(rx[i], x);
    if (c < p.d) {
      float w[VE], b[VE], g[VE];
      if (p.post_weight) R::load_f32(p.post_weight, c, w);
      if (p.post_bias) R::load_f32(p.post_bias, c, b);
      if (p.gate_kind == MOE_BLOCK_GATE_CHANNEL) R::load_f32(p.gate, c, g);
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        float v = n[i][j];
        if (p.post_weight) v = v * r * w[j] + (p.post_bias ? b[j] : 0.f);
        if (p.gate_kind == MOE_BLOCK_GATE_CHANNEL) v *= g[j];
        n[i][j] = (float)from_f32<E>(x[j] + ag * v);
      }
      store16_f32(xo + c, n[i]);
    }
  }
  if (!p.u) return;
  center<R, W, NV>(a, n, buf, flip, mu, r);
  if (first) {
    p.pre_mean[t] = mu;
    p.pre_rstd[t] = r;
  }
  E* u = static_cast<E*>(p.u) + (size_t)t * p.d;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = R::col(i);
    if (c < p.d) {
      float w[VE], b[VE];
      R::load_f32(p.pre_weight, c, w);
      if (p.pre_bias) R::load_f32(p.pre_bias, c, b);
#pragma unroll
      for (int j = 0; j < VE; ++j) n[i][j] = n[i][j] * r * w[j] + (p.pre_bias ? b[j] : 0.f);
      store16_f32(u + c, n[i]);
    }
  }
}

// Rows of up to 8 values a lane, backward.  A block's groups take rows as in the forward; the
// next rows' arrays come by DMA into LDS (16 KB of bf16 a row of 2048, no registers; where LDS holds one
// round alone, fp32 rows past 4096: once it has been read).  Weights stay in registers: a load of them in the
// loop would wait for the DMA before it.
// One block a CU (a second one's partial rows cost more than it hides: 8192 x 2048 48 -> 55 us).
// Instead of this, a block of four waves for each row, the next one's loads in registers: 8192 x 2048 58
// us, 16384 x 4096 188 (now 155).
// PRE, POST: the norms that there are.
template <class E, int W, int NV, bool PRE, bool POST>
__global__ __launch_bounds__(64 * row_block_waves(W), 4) void block_norm_bwd_kernel(BlockArgs a) {
  using R = Row<E, W, NV>;
  constexpr int VE = R::VE, BW = row_block_waves(W), GROUPS = BW / W, WAVE = 4 * NV * 1024;
  constexpr int DEPTH = BW * WAVE > 65536 ? 1 : 2;
  __shared__ __attribute__((aligned(16))) char ring[DEPTH][BW][WAVE];
  __shared__ float buf[GROUPS][6][W];
  const moe_block_norm& p = a.p;
  const bool channel = p.gate_kind == MOE_BLOCK_GATE_CHANNEL;
  const bool token = p.gate_kind == MOE_BLOCK_GATE_TOKEN;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int group = wave / W, wr = wave % W;
  const int step = gridDim.x * GROUPS;
  float s[kSums][NV][VE], wpre[NV][VE], wpost[NV][VE], bpost[NV][VE], g[NV][VE];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      s[0][i][j] = s[1][i][j] = s[2][i][j] = s[3][i][j] = 0.f;
      wpre[i][j] = wpost[i][j] = bpost[i][j] = 0.f;
      g[i][j] = 1.f;
    }
    if (R::col(i) < p.d) {
      if (PRE) R::load_f32(p.pre_weight, R::col(i), wpre[i]);
      if (POST) R::load_f32(p.post_weight, R::col(i), wpost[i]);
      if (POST && p.post_bias) R::load_f32(p.post_bias, R::col(i), bpost[i]);
      if (channel) R::load_f32(p.gate, R::col(i), g[i]);
    }
  }
  const int bytes = p.d * (int)sizeof(E);
  float nmx = 0.f, nrx = 0.f, nmf = 0.f, nrf = 0.f, ng = 1.f;
  // (rows past the last read zeros, with means of zero: they add zeros)
  auto fetch = [&](int t, char* dst) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (what was there has been read)
    const int n = t < p.T ? bytes : 0;
    const size_t at = t < p.T ? (size_t)t * p.d : 0;
    if constexpr (PRE) {
      dma_row<W, NV>(static_cast<const E*>(p.du) + at, n, wr, dst);
      dma_row<W, NV>(static_cast<const E*>(p.x_out) + at, n, wr, dst + NV * 1024);
    }
    dma_row<W, NV>(static_cast<const E*>(p.f) + at, n, wr, dst + 2 * NV * 1024);
    if (p.dres) dma_row<W, NV>(static_cast<const E*>(p.dres) + at, n, wr, dst + 3 * NV * 1024);
    const int q = min(t, p.T - 1);
    if constexpr (PRE) {
      nmx = p.pre_mean[q];
      nrx = p.pre_rstd[q];
    }
    if constexpr (POST) {
      nmf = p.post_mean[q];
      nrf = p.post_rstd[q];
    }
    if (token) ng = p.gate[q];
  };
  auto read = [&](const char* src, int k, int i, float* out) {
    R::unpack(*reinterpret_cast<const u32x4_t*>(src + (k * NV + i) * 1024 + lane * 16), out);
  };
  int flip = 0, cur = 0;
  float (*sums)[W] = buf[group];
  const int first = blockIdx.x * GROUPS;
  if (first < p.T) fetch(first + group, ring[0][wave]);
  for (int t0 = first; t0 < p.T; t0 += step) {  // (the same rounds in all waves)
    const int t = t0 + group;
    const bool there = t < p.T;
    // These rows have landed, and their statistics: all that the wave has in flight, with the last rows' stores,
    // as how many of them are newer than the DMA goes by the form, the ring's depth and the round
    asm volatile("s_waitcnt vmcnt(0)" : "+v"(nmx), "+v"(nrx), "+v"(nmf), "+v"(nrf), "+v"(ng)::"memory");
    const float mx = nmx, rx = nrx, mf = nmf, rf = nrf, ag = p.scale * ng;
    const char* src = ring[cur][wave];
    if constexpr (DEPTH == 2) {
      cur ^= 1;
      if (t0 + step < p.T) fetch(t + step, ring[cur][wave]);
    }
    float G[NV][VE];
    // ---- the pre-norm's backward: G
    if constexpr (PRE) {
      float xh[NV][VE], q[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        // past the row's end x, du and w are zeros, and the mean is taken as zero: every sum is
        const float m = there && R::col(i) < p.d ? mx : 0.f;
        read(src, 1, i, xh[i]);
        read(src, 0, i, G[i]);
#pragma unroll
        for (int j = 0; j < VE; ++j) {
          xh[i][j] = (xh[i][j] - m) * rx;
          s[0][i][j] += G[i][j] * xh[i][j];
          s[1][i][j] += G[i][j];
          G[i][j] *= wpre[i][j];
          q[0] += G[i][j];
          q[1] += G[i][j] * xh[i][j];
        }
      }
      all_sums<W>(q, sums, flip);
      const float m0 = q[0] * a.inv_d, m1 = q[1] * a.inv_d;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const bool in = R::col(i) < p.d;
        float res[VE] = {};
        if (p.dres) read(src, 3, i, res);
#pragma unroll
        for (int j = 0; j < VE; ++j) G[i][j] = in ? res[j] + rx * (G[i][j] - m0 - xh[i][j] * m1) : 0.f;
      }
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i) read(src, 3, i, G[i]);
    }
    E* dx = static_cast<E*>(p.dx) + (size_t)t * p.d;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (there && R::col(i) < p.d) store16_f32(dx + R::col(i), G[i]);
    // ---- the gate and the post norm: G becomes dn (times w_post)
    float fh[NV][VE], q[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const float m = POST && there && R::col(i) < p.d ? mf : 0.f;
      read(src, 2, i, fh[i]);
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        if constexpr (POST) fh[i][j] = (fh[i][j] - m) * rf;
        if (token) q[2] += G[i][j] * (POST ? fh[i][j] * wpost[i][j] + bpost[i][j] : fh[i][j]);
        G[i][j] *= ag;
        s[2][i][j] += G[i][j] * fh[i][j];
        s[3][i][j] += G[i][j];
        G[i][j] *= g[i][j];
        if constexpr (POST) {
          G[i][j] *= wpost[i][j];
          q[0] += G[i][j];
          q[1] += G[i][j] * fh[i][j];
        }
      }
    }
    if (DEPTH == 1 && t0 + step < p.T) fetch(t + step, ring[0][wave]);  // (all of these rows is read)
    // (two buffers in turn: the pre-norm's sums took the first)
    if (token) all_sums<W>(q, sums, flip);
    else if (POST) all_sums<W>(reinterpret_cast<float (&)[2]>(q), sums, flip);
    if (token && there && wr == 0 && lane == 0) p.d_gate[t] = p.scale * q[2];
    const float m0 = q[0] * a.inv_d, m1 = q[1] * a.inv_d;
    E* df = static_cast<E*>(p.df) + (size_t)t * p.d;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (there && R::col(i) < p.d) {
        if constexpr (POST)
#pragma unroll
          for (int j = 0; j < VE; ++j) G[i][j] = rf * (G[i][j] - m0 - fh[i][j] * m1);
        store16_f32(df + R::col(i), G[i]);
      }
  }
  // the block's partial row: the groups' sums are added in order through LDS
  float* part = a.part + (size_t)blockIdx.x * kSums * p.d;
  if constexpr (GROUPS > 1) {
    float* cols = reinterpret_cast<float*>(ring);  // [4][d]
    static_assert(sizeof(ring) >= (size_t)kSums * 64 * W * NV * VE * sizeof(float), "the ring holds a row of sums");
    for (int k = 0; k < GROUPS; ++k) {
      __syncthreads();
      if (group == k)
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int c = R::col(i);
          if (c < p.d)
#pragma unroll
            for (int q = 0; q < kSums; ++q)
#pragma unroll
              for (int j = 0; j < VE; ++j)
                cols[q * p.d + c + j] = (k ? cols[q * p.d + c + j] : 0.f) + s[q][i][j];
        }
    }
    __syncthreads();
    for (int c = threadIdx.x * 4; c < kSums * p.d; c += 64 * BW * 4)
      *reinterpret_cast<f32x4_t*>(part + c) = *reinterpret_cast<const f32x4_t*>(cols + c);
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = R::col(i);
      if (c < p.d)
#pragma unroll
        for (int k = 0; k < kSums; ++k)
#pragma unroll
          for (int j = 0; j < VE; j += 4)
            *reinterpret_cast<f32x4_t*>(part + (size_t)k * p.d + c + j) =
                f32x4_t{s[k][i][j], s[k][i][j + 1], s[k][i][j + 2], s[k][i][j + 3]};
    }
  }
}

// Wide rows, 16 values a lane of a block of sixteen waves: two of the column sums are held in LDS,
// where every lane has its own columns (in registers they spill), and nothing is fetched ahead.
template <class E, bool PRE, bool POST>
__global__ __launch_bounds__(1024) void block_norm_bwd_wide_kernel(BlockArgs a) {
  constexpr int W = 16, VE = Vec16<E>::N, NV = 16 / VE;
  using R = Row<E, W, NV>;
  __shared__ float buf[6][W];
  __shared__ f32x4_t lds[2 * 4 * 1024];  // [2][NV VE / 4][1024]: a lane's sums 0 and 1
  const moe_block_norm& p = a.p;
  const bool channel = p.gate_kind == MOE_BLOCK_GATE_CHANNEL;
  const bool token = p.gate_kind == MOE_BLOCK_GATE_TOKEN;
  auto own = [&](int k, int i, int j) -> f32x4_t& {  // values j .. j + 3 of vector i of sum k
    return lds[(k * 4 + (i * VE + j) / 4) * 1024 + threadIdx.x];
  };
  float s[2][NV][VE];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      s[0][i][j] = s[1][i][j] = 0.f;
      if (j % 4 == 0) own(0, i, j) = own(1, i, j) = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
  int flip = 0;
  for (int t = blockIdx.x; t < p.T; t += gridDim.x) {
    float G[NV][VE];
    const float ag = token ? p.scale * p.gate[t] : p.scale;
    if constexpr (PRE) {
      u32x4_t nu[NV], nx[NV];
      R::load(p.du, t, p.d, nu);
      R::load(p.x_out, t, p.d, nx);
      const float mx = p.pre_mean[t], rx = p.pre_rstd[t];
      float q[2] = {0.f, 0.f}, xh[NV][VE];
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const bool in = R::col(i) < p.d;
        const float m = in ? mx : 0.f;
        float w[VE] = {};
        if (in) R::load_f32(p.pre_weight, R::col(i), w);
        R::unpack(nx[i], xh[i]);
        R::unpack(nu[i], G[i]);
#pragma unroll
        for (int j = 0; j < VE; j += 4) {
          f32x4_t s0 = own(0, i, j), s1 = own(1, i, j);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float &x = xh[i][j + e], &v = G[i][j + e];
            x = (x - m) * rx;
            s0[e] += v * x;
            s1[e] += v;
            v *= w[j + e];
            q[0] += v;
            q[1] += v * x;
          }
          own(0, i, j) = s0;
          own(1, i, j) = s1;
        }
      }
      u32x4_t nr[NV];
      if (p.dres) R::load(p.dres, t, p.d, nr);
      all_sums<W>(q, buf, flip);
      const float m0 = q[0] * a.inv_d, m1 = q[1] * a.inv_d;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const bool in = R::col(i) < p.d;
        float res[VE] = {};
        if (p.dres) R::unpack(nr[i], res);
#pragma unroll
        for (int j = 0; j < VE; ++j) G[i][j] = in ? res[j] + rx * (G[i][j] - m0 - xh[i][j] * m1) : 0.f;
      }
    } else {
      u32x4_t nr[NV];
      R::load(p.dres, t, p.d, nr);
#pragma unroll
      for (int i = 0; i < NV; ++i) R::unpack(nr[i], G[i]);
    }
    u32x4_t nf[NV];
    R::load(p.f, t, p.d, nf);
    E* dx = static_cast<E*>(p.dx) + (size_t)t * p.d;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (R::col(i) < p.d) store16_f32(dx + R::col(i), G[i]);
    const float mf = POST ? p.post_mean[t] : 0.f, rf = POST ? p.post_rstd[t] : 0.f;
    float fh[NV][VE], q[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = R::col(i);
      const bool in = c < p.d;
      float w[VE] = {}, b[VE] = {}, g[VE] = {};
      if (in) {
        if (POST) R::load_f32(p.post_weight, c, w);
        if (POST && token && p.post_bias) R::load_f32(p.post_bias, c, b);
        if (channel) R::load_f32(p.gate, c, g);
      }
      const float m = POST && in ? mf : 0.f;
      R::unpack(nf[i], fh[i]);
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        if constexpr (POST) fh[i][j] = (fh[i][j] - m) * rf;
        if (token) q[2] += G[i][j] * (POST ? fh[i][j] * w[j] + b[j] : fh[i][j]);
        G[i][j] *= ag;
        s[0][i][j] += G[i][j] * fh[i][j];
        s[1][i][j] += G[i][j];
        if (channel) G[i][j] *= g[j];
        if constexpr (POST) {
          G[i][j] *= w[j];
          q[0] += G[i][j];
          q[1] += G[i][j] * fh[i][j];
        }
      }
    }
    if (token) all_sums<W>(q, buf, flip);
    else if (POST) all_sums<W>(reinterpret_cast<float (&)[2]>(q), buf, flip);
    if (token && threadIdx.x == 0) p.d_gate[t] = p.scale * q[2];
    const float m0 = q[0] * a.inv_d, m1 = q[1] * a.inv_d;
    E* df = static_cast<E*>(p.df) + (size_t)t * p.d;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (R::col(i) < p.d) {
        if constexpr (POST)
#pragma unroll
          for (int j = 0; j < VE; ++j) G[i][j] = rf * (G[i][j] - m0 - fh[i][j] * m1);
        store16_f32(df + R::col(i), G[i]);
      }
  }
  float* part = a.part + (size_t)blockIdx.x * kSums * p.d;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = R::col(i);
    if (c < p.d)
#pragma unroll
      for (int j = 0; j < VE; j += 4) {
        *reinterpret_cast<f32x4_t*>(part + c + j) = own(0, i, j);
        *reinterpret_cast<f32x4_t*>(part + (size_t)p.d + c + j) = own(1, i, j);
#pragma unroll
        for (int k = 0; k < 2; ++k)
          *reinterpret_cast<f32x4_t*>(part + (size_t)(2 + k) * p.d + c + j) =
              f32x4_t{s[k][i][j], s[k][i][j + 1], s[k][i][j + 2], s[k][i][j + 3]};
      }
  }
}

// The weights' gradients from the n partial rows [n][4][d]: a block takes 16 columns of the four
// sums, sixteen threads (16 bytes each) by 64 shares of the partials (bound by their latency: 256 partials of
// d = 4096, 16 MB, 7 us).
constexpr int kDwShares = 64;
__global__ __launch_bounds__(16 * kDwShares) void block_norm_dw_kernel(BlockArgs a, int n) {
  const moe_block_norm& p = a.p;
  constexpr int G = 8;
  __shared__ f32x4_t sum[kDwShares][16];
  const int l = threadIdx.x & 15, sh = threadIdx.x >> 4;
  const int q = l & 3, c = (blockIdx.x * 4 + q) * 4;
  f32x4_t s = {0.f, 0.f, 0.f, 0.f};
  if (c < p.d) {
    const float* at = a.part + (size_t)(l >> 2) * p.d + c;
#pragma unroll 8
    for (int i = sh; i < n; i += kDwShares) s += *reinterpret_cast<const f32x4_t*>(at + (size_t)i * kSums * p.d);
  }
  sum[sh][l] = s;
  __syncthreads();
  if (sh < G) {
    for (int i = sh + G; i < kDwShares; i += G) s += sum[i][l];
    sum[sh][l] = s;  // (read by this thread alone so far)
  }
  __syncthreads();
  if (sh == 0) {
    for (int i = 1; i < G; ++i) s += sum[i][l];
    sum[0][l] = s;
  }
  __syncthreads();
  f32x4_t tot[kSums];
#pragma unroll
  for (int k = 0; k < kSums; ++k) tot[k] = sum[0][4 * k + q];
  if (threadIdx.x >= 4 || c >= p.d) return;
  auto put = [&](float* out, f32x4_t v) {
    if (!out) return;
    f32x4_t* o = reinterpret_cast<f32x4_t*>(out + c);
    *o = p.accumulate ? *o + v : v;
  };
  const f32x4_t s3 = tot[2], s4 = tot[3];
  if (p.pre_weight) {
    put(p.d_pre_weight, tot[0]);
    put(p.d_pre_bias, tot[1]);
  }
  if (p.gate_kind == MOE_BLOCK_GATE_CHANNEL) {
    f32x4_t w = {1.f, 1.f, 1.f, 1.f}, b = {0.f, 0.f, 0.f, 0.f};
    if (p.post_weight) w = *reinterpret_cast<const f32x4_t*>(p.post_weight + c);
    if (p.post_bias) b = *reinterpret_cast<const f32x4_t*>(p.post_bias + c);
    const f32x4_t g = *reinterpret_cast<const f32x4_t*>(p.gate + c);
    put(p.d_gate, w * s3 + b * s4);
    if (p.post_weight) {
      put(p.d_post_weight, g * s3);
      put(p.d_post_bias, g * s4);
    }
  } else if (p.post_weight) {
    put(p.d_post_weight, s3);
    put(p.d_post_bias, s4);
  }
}

// Waves per row: the fewest with a vector in each lane (more rows in a block, and fewer barriers between
// waves), two of fp32 past sixteen waves' reach; 32: the wide kernels.
int row_waves(int d, int ve) {
  for (int W : {1, 2, 4, 8, 16})
    if (vectors(d, ve, W) <= 1) return W;
  return vectors(d, ve, 16) * ve <= 8 ? 16 : 32;
}

int blocks_bwd(int T, int d, int ve) {
  const int W = row_waves(d, ve), rows = W > 16 ? 1 : row_block_waves(W) / W;
  return std::min(ceil_div(T, rows), num_cus());
}

template <class E, bool PRE, bool POST>
void fwd(const BlockArgs& a, int W, hipStream_t s) {
  constexpr int VE = Vec16<E>::N;
  const int blocks = std::min(ceil_div(a.p.T, row_block_waves(W) / W), (W == 16 ? 1 : 3) * num_cus());
#define BLOCK_FWD(W_, NV_)                                                    \
  MOE_TIMED("block_norm_fwd", s, block_norm_fwd_kernel<E, W_, NV_, PRE, POST> \
            <<<blocks, 64 * row_block_waves(W_), 0, s>>>(a))
  if (W == 1) BLOCK_FWD(1, 1);
  else if (W == 2) BLOCK_FWD(2, 1);
  else if (W == 4) BLOCK_FWD(4, 1);
  else if (W == 8) BLOCK_FWD(8, 1);
  else if (vectors(a.p.d, VE, 16) == 1) BLOCK_FWD(16, 1);
  else if constexpr (VE == 4) BLOCK_FWD(16, 2);
#undef BLOCK_FWD
}

template <class E>
hipError_t fwd(const BlockArgs& a, hipStream_t s) {
  const moe_block_norm& p = a.p;
  const int W = row_waves(p.d, Vec16<E>::N), most = rows_per_launch(16);
  if (p.T > 0 && W <= 16) {
    if (!p.pre_weight) fwd<E, false, true>(a, W, s);
    else if (p.post_weight) fwd<E, true, true>(a, W, s);
    else fwd<E, true, false>(a, W, s);
    return hipGetLastError();
  }
  for (int t = 0; t < p.T; t += most) {  // (wide rows: a block each)
    BlockArgs part = a;
    moe_block_norm& q = part.p;
    const size_t at = (size_t)t * p.d;
    q.x = static_cast<const E*>(p.x) + at;
    q.f = static_cast<const E*>(p.f) + at;
    q.x_out = static_cast<E*>(p.x_out) + at;
    if (p.u) q.u = static_cast<E*>(p.u) + at;
    for (float** v : {&q.post_mean, &q.post_rstd, &q.pre_mean, &q.pre_rstd})
      if (*v) *v += t;
    if (p.gate && p.gate_kind == MOE_BLOCK_GATE_TOKEN) q.gate += t;
    q.T = std::min(p.T - t, most);
    MOE_TIMED("block_norm_fwd", s, block_norm_fwd_wide_kernel<E><<<q.T, 1024, 0, s>>>(part));
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <class E, bool PRE, bool POST>
void bwd(const BlockArgs& a, int blocks, hipStream_t s) {
  constexpr int VE = Vec16<E>::N;
  const int W = row_waves(a.p.d, VE);
#define BLOCK_BWD(W_, NV_)                                                    \
  MOE_TIMED("block_norm_bwd", s, block_norm_bwd_kernel<E, W_, NV_, PRE, POST> \
            <<<blocks, 64 * row_block_waves(W_), 0, s>>>(a))
  if (W == 1) BLOCK_BWD(1, 1);
  else if (W == 2) BLOCK_BWD(2, 1);
  else if (W == 4) BLOCK_BWD(4, 1);
  else if (W == 8) BLOCK_BWD(8, 1);
  else if (W == 16 && vectors(a.p.d, VE, 16) == 1) BLOCK_BWD(16, 1);
  else if (W == 16) {
    if constexpr (VE == 4) BLOCK_BWD(16, 2);
  } else
    MOE_TIMED("block_norm_bwd", s, block_norm_bwd_wide_kernel<E, PRE, POST><<<blocks, 1024, 0, s>>>(a));
#undef BLOCK_BWD
}

template <class E>
void bwd(const BlockArgs& a, int blocks, hipStream_t s) {
  if (!a.p.pre_weight) bwd<E, false, true>(a, blocks, s);
  else if (a.p.post_weight) bwd<E, true, true>(a, blocks, s);
  else bwd<E, true, false>(a, blocks, s);
}

}  // namespace

hipError_t launch_block_norm_fwd(const moe_block_norm* p, hipStream_t s) {
  BlockArgs a{*p, nullptr, 1.0f / (float)p->d};
  return p->dtype == MOE_BF16 ? fwd<bf16_t>(a, s) : fwd<float>(a, s);
}

size_t block_norm_ws_bytes(int T, int d, int bf16) {
  return (size_t)blocks_bwd(T, d, bf16 ? 8 : 4) * kSums * d * sizeof(float);
}

hipError_t launch_block_norm_bwd(const moe_block_norm* p, hipStream_t s) {
  const bool bf16 = p->dtype == MOE_BF16;
  BlockArgs a{*p, static_cast<float*>(p->ws), 1.0f / (float)p->d};
  const int blocks = blocks_bwd(p->T, p->d, bf16 ? 8 : 4);
  if (p->T > 0) {
    bf16 ? bwd<bf16_t>(a, blocks, s) : bwd<float>(a, blocks, s);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  MOE_TIMED("block_norm_dw", s,
            block_norm_dw_kernel<<<ceil_div(p->d, 16), 16 * kDwShares, 0, s>>>(a, blocks));
  return hipGetLastError();
}

}  // namespace moe
