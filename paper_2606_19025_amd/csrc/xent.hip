// Softmax cross entropy of a linear head over a vocabulary, without keeping the logits.
//
//   z_tv = scale x_t . w_v;   lse_t = log sum_v exp z_tv;   loss_t = lse_t - z_ty + z_coef lse_t^2
//   dz_tv = g_t ((1 + 2 z_coef lse_t) exp(z_tv - lse_t) - [v = y_t])
//   dx = scale dz W,  dW = scale dz^T x
// The scale, and the mean's 1 / n where that is all of g, are factors of dx and dW at their ends (out), so
// that dz's roundings do not take them in: -1 of a label's word is exact, not off by one part in up to 2^8
// in all tokens alike.
//
// Four products of 2 N V d operations (gemm.hip, gemm_tile.hip: XE_* kinds).  Forward: a tile of
// logits ends in (max, sum of 2^(z - max)) of each of its rows, and the label's logit where it is
// among its columns; a second launch joins the pieces of a row.  Backward, for one piece of the
// vocabulary after the other: the logits again, which end as dz in dtype, then dx and dW of the
// piece in one launch.  dx is summed over pieces (and parts of K) in fp32 and rounded once.
//
// Tokens that do not count (label < 0) are left out of every product (but the forward's of up to kFew
// tokens): the others' rows are copied together first (where all count, x itself is read), so a padded
// batch costs what its tokens do, and nothing that stands in a padded row enters a gradient.  How many there
// are stays on the device, as in the dispatch.
//
// Bound by the matrix units with many tokens (8192, d = 2048, 49152 words, bf16: forward 1.29 ms, 1.28 PFLOP/s,
// backward 3.91 ms, 1.27 over its three products; of a library's product of the logits' size alone 1.24) and
// by the streams of W and dW with few (24 tokens forward 49 us, of which W at a copy's rate 41; backward 144,
// where W is read twice and dW written).
// dz is rounded to bf16, as the matrix instructions take it; what of it is a token's, and not its words', stays
// out of that where it can (above, Plan::two and Plan::fold): dx is off by 0.0017 of its norm, a bf16
// output's own rounding, dW by that for a mean and for few tokens, and by 0.0024 for gradients of the tokens' own.
#include <algorithm>
#include <cmath>

#include "gemm.h"
#include "kernels.h"
#include "timing.h"

namespace moe {
namespace {

constexpr int kCountRows = 1024;  // tokens of a counting block
constexpr int kDirect = 8192;     // up to here every block counts all labels itself
constexpr int kLossThreads = 1024;
constexpr int kFew = 256;         // up to here, a large tile's rows, the forward leaves out none
constexpr int kTwo = 32;          // up to here the backward keeps dz in two values (Plan::two)

struct RowArgs {
  const void* x;
  const int32_t* label;
  const float* lse;    // backward
  const float* dloss;  // backward, or NULL: 1 / the number of tokens that count
  int N, d, V, size;   // size: bytes of an element
  float scale;
  int* count;          // [blocks of kCountRows]
  int* pos;            // [N] row of a token among those that count, or -1
  int* off;            // {0, tokens that count, 0, twice them}
  int two;             // backward: a token's row is copied twice, in any case
  int fold;            // backward: the gradients dloss go into xs and factor (Plan::fold)
  const void* w;       // (fold)
  float z2;
  void* xs;
  float* factor;       // of a row of dx, by row
  int* row_label;      // the rest by row
  float* row_lse;      // backward
  float* coef;
  float* out;
  void* xc;
  int* counters;       // backward: cleared for the launches that follow
  int n_counters;
};

DEVI int block_sum_256(int v, int* buf) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
  __syncthreads();
  return buf[0] + buf[1] + buf[2] + buf[3];
}

__global__ __launch_bounds__(256) void xent_count_kernel(const int32_t* label, int N, int* count) {
  __shared__ int buf[4];
  int v = 0;
  for (int i = threadIdx.x; i < kCountRows; i += 256) {
    const int t = blockIdx.x * kCountRows + i;
    v += t < N && label[t] >= 0;
  }
  v = block_sum_256(v, buf);
  if (threadIdx.x == 0) count[blockIdx.x] = v;
}

// The rows of the tokens that count, R tokens a block: 4 up to 4096 of them, for more rows in flight
// (measured, a quarter left out, 16 and 4 a block: 1000 of d = 4096 14 and 7 us, 1531 of 768 6.4 and 5.4), 16
// for more, as every block reads the labels (8000 of d = 256 6.5 and 7.2 us).
template <bool BWD, int R>
__global__ __launch_bounds__(256) void xent_rows_kernel(RowArgs a) {
  __shared__ int buf[4];
  __shared__ int row[R];
  __shared__ int word[BWD ? R : 1];
  __shared__ float2 given[BWD ? R : 1];  // lse and dloss
  const int t0 = blockIdx.x * R;
  // tokens that count before this block's, and all of them
  int before = 0, total = 0;
  if (a.N <= kDirect) {
#pragma unroll 8
    for (int t = threadIdx.x; t < a.N; t += 256) {
      const int v = a.label[t] >= 0;
      total += v;
      before += t < t0 ? v : 0;
    }
  } else {
    const int first = t0 / kCountRows;
    for (int b = threadIdx.x; b < ceil_div(a.N, kCountRows); b += 256) {
      total += a.count[b];
      before += b < first ? a.count[b] : 0;
    }
    for (int t = first * kCountRows + threadIdx.x; t < t0; t += 256) before += a.label[t] >= 0;
  }
  before = block_sum_256(before, buf);
  total = block_sum_256(total, buf);
  if (threadIdx.x < 64) {
    const int t = t0 + threadIdx.x;
    const int y = (int)threadIdx.x < R && t < a.N ? a.label[t] : -1;
    const unsigned long long counts = __ballot(y >= 0);
    const int p = y < 0 ? -1 : before + __builtin_popcountll(counts & ((1ull << threadIdx.x) - 1));
    if ((int)threadIdx.x < R) {
      row[threadIdx.x] = p;
      if (t < a.N) a.pos[t] = p;
    }
    if (p >= 0) {
      a.row_label[p] = y;
      if constexpr (BWD) {
        a.row_lse[p] = a.lse[t];
        // (a label that is no word of the vocabulary makes what it enters NaN)
        const float g = a.dloss ? a.dloss[t] : 1.0f;
        if (!a.fold) a.coef[p] = y < a.V ? g : NAN;
        word[threadIdx.x] = y;
        given[threadIdx.x] = float2{a.lse[t], g};
      }
    }
    if (blockIdx.x == 0 && threadIdx.x < 4)
      a.off[threadIdx.x] = threadIdx.x & 1 ? total * (1 + (threadIdx.x >> 1)) : 0;
  }
  if (BWD && blockIdx.x == 0 && threadIdx.x == 0)
    *a.out = a.dloss ? a.scale : total ? a.scale / (float)total : 0.0f;
  if (BWD && blockIdx.x == 0)
    for (int i = threadIdx.x; i < a.n_counters; i += 256) a.counters[i] = 0;
  if (total == a.N && !a.two && !a.fold) return;  // x itself is read
  __syncthreads();
  // 256 / R threads to a row, so that all rows' loads are in flight
  const int chunks = a.d * a.size / 16;
  const int r = threadIdx.x / (256 / R), p = row[r];
  if (p < 0) return;
  const u32x4_t* src = static_cast<const u32x4_t*>(a.x) + (size_t)(t0 + r) * chunks;
  if constexpr (BWD) {
    if (a.fold) {
      // the label's entry of dz, but for the gradient: q = (1 + 2 z_coef lse) exp(z - lse) - 1
      const int y = word[r];
      const float lse = given[r].x, g = given[r].y;
      const bf16_t* x = static_cast<const bf16_t*>(a.x) + (size_t)(t0 + r) * a.d;
      const bf16_t* w = static_cast<const bf16_t*>(a.w) + (size_t)(y < a.V ? y : 0) * a.d;
      float dot = 0.0f;
#pragma unroll 2
      for (int c = threadIdx.x % (256 / R); c < chunks; c += 256 / R) {
        float u[8], v[8];
        load16_f32(x + 8 * c, u);
        load16_f32(w + 8 * c, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) dot += u[e] * v[e];
      }
#pragma unroll
      for (int o = 128 / R; o > 0; o >>= 1) dot += __shfl_xor(dot, o, 64);
      float q = (1.0f + a.z2 * lse) * expf(a.scale * dot - lse) - 1.0f;
      if (!(fabsf(q) >= 0x1p-8f && fabsf(q) <= 0x1p8f)) q = 1.0f;  // (any factor is right)
      if (threadIdx.x % (256 / R) == 0) {
        a.coef[p] = y < a.V ? 1.0f / q : NAN;
        a.factor[p] = g * q;
      }
      bf16_t* xs = static_cast<bf16_t*>(a.xs) + (size_t)p * a.d;
      bf16_t* xc = static_cast<bf16_t*>(a.xc) + (size_t)p * a.d;
#pragma unroll 2
      for (int c = threadIdx.x % (256 / R); c < chunks; c += 256 / R) {
        float u[8];
        load16_f32(x + 8 * c, u);
        if (total < a.N) store16_f32(xc + 8 * c, u);
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] *= g * q;
        store16_f32(xs + 8 * c, u);
      }
      return;
    }
  }
  u32x4_t* dst = static_cast<u32x4_t*>(a.xc) + (size_t)(a.two ? 2 * p : p) * chunks;
  u32x4_t* again = dst + (a.two ? chunks : 0);
#pragma unroll 4
  for (int c = threadIdx.x % (256 / R); c < chunks; c += 256 / R) {
    const u32x4_t v = src[c];
    dst[c] = v;
    if (a.two) again[c] = v;
  }
}

// (max, sum) pairs of base 2 joined.  (fmaxf leaves a NaN out: the sums carry it on)
DEVI float2 join(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x);
  if (m == -INFINITY) return float2{m, a.y + b.y};
  return float2{m, a.y * __builtin_amdgcn_exp2f(a.x - m) + b.y * __builtin_amdgcn_exp2f(b.x - m)};
}

// lse and loss of R tokens a block from their P partials, 1024 / R threads a token.  Few tokens a block
// where there are few: 24 tokens of 1536 partials took 42 us with 64 a block.  pos: the tokens' rows, or
// NULL: their own numbers.  The block that ends last adds the blocks' sums of losses and tokens, in order.
template <int R>
__global__ __launch_bounds__(kLossThreads) void xent_loss_kernel(
    int N, int V, int P, float z_coef, const int* label, const int* pos, const float2* part,
    const float* z_label, float* loss, float* lse, double* sums, int* done, float* total) {
  constexpr int S = kLossThreads / R, WAVES = kLossThreads / 64;
  __shared__ float2 seg[WAVES][R];
  __shared__ bool last;
  const int r = threadIdx.x % R, q = threadIdx.x / R;
  const int t = blockIdx.x * R + r;
  const int y = t < N ? label[t] : -1;
  const int p = y < 0 ? -1 : pos ? pos[t] : t;
  float2 v = {-INFINITY, 0.f};
  if (p >= 0) {
#pragma unroll 4
    for (int i = q; i < P; i += S) v = join(v, part[(size_t)i * N + p]);
  }
  // the threads of a token in a wave are R lanes apart; then the waves'
  auto across = [&]() {
#pragma unroll
    for (int o = R; o < 64; o *= 2) v = join(v, float2{__shfl_xor(v.x, o, 64), __shfl_xor(v.y, o, 64)});
  };
  across();
  if ((threadIdx.x & 63) < R) seg[threadIdx.x >> 6][r] = v;
  __syncthreads();
  float out = 0.f;
  if (threadIdx.x < 64) {
    v = float2{-INFINITY, 0.f};
#pragma unroll
    for (int w = threadIdx.x / R; w < WAVES; w += 64 / R) v = join(v, seg[w][r]);
    across();
    if ((int)threadIdx.x < R && t < N) {
      float l = 0.f;
      if (p >= 0) {
        l = v.x * kLn2 + logf(v.y);
        out = y < V ? l - z_label[p] + z_coef * l * l : NAN;
      }
      lse[t] = l;
      loss[t] = out;
    }
    const int counted = __builtin_popcountll(__ballot((int)threadIdx.x < R && y >= 0));
    double s = (double)out;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if (threadIdx.x == 0) {
      __hip_atomic_store(sums + 2 * blockIdx.x, s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(sums + 2 * blockIdx.x + 1, (double)counted, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      last = __hip_atomic_fetch_add(done, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
    }
  }
  __syncthreads();
  if (!last || threadIdx.x >= 64) return;
  // (even lanes the losses, odd ones the tokens)
  double s = 0.0;
  for (int i = threadIdx.x; i < 2 * (int)gridDim.x; i += 64)
    s += __hip_atomic_load(sums + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
  for (int o = 32; o > 1; o >>= 1) s += __shfl_xor(s, o, 64);
  if (threadIdx.x < 2) total[threadIdx.x] = (float)s;
}

// total of no tokens.
__global__ __launch_bounds__(64) void xent_none_kernel(float* total) {
  if (threadIdx.x < 2) total[threadIdx.x] = 0.f;
}

// n 16-byte pieces of zeros (the gradient of no tokens).
__global__ __launch_bounds__(256) void xent_clear_kernel(u32x4_t* p, size_t n) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256)
    p[i] = u32x4_t{0u, 0u, 0u, 0u};
}

// dx[t] = the sum of its row's (TWO: both rows') S partial sums, or zeros.  SH threads share a vector's
// partials, whose sums are added in order: where the vectors are few and the partials many (5 tokens, d =
// 768, 192 partials 8 us, with eight 5).
template <class E, int SH, bool TWO>
__global__ __launch_bounds__(256) void xent_dx_kernel(E* dx, const int* pos, const float* part, size_t stride,
                                                      int S, int N, int d, const float* out,
                                                      const float* factor) {
  constexpr int V = Vec16<E>::N, AT = 256 / SH;
  __shared__ float sum[SH > 1 ? SH : 1][SH > 1 ? AT : 1][V + 4];
  const int chunks = d / V, sh = threadIdx.x / AT, l = threadIdx.x % AT;
  const size_t n = (size_t)N * chunks;
  // (every thread of a block takes the same rounds)
  for (size_t i0 = (size_t)blockIdx.x * AT; i0 < n; i0 += (size_t)gridDim.x * AT) {
    const size_t i = i0 + l;
    const int t = (int)(i / chunks), c = (int)(i % chunks) * V;
    const int p = i < n ? pos[t] : -1;
    float v[V] = {};
    if (p >= 0) {
      const float* q = part + (size_t)(TWO ? 2 * p : p) * d + c;
#pragma unroll 4
      for (int s = sh; s < S; s += SH) {
#pragma unroll
        for (int j = 0; j < V; j += 4) {
          f32x4_t u = *reinterpret_cast<const f32x4_t*>(q + s * stride + j);
          if (TWO) u += *reinterpret_cast<const f32x4_t*>(q + s * stride + d + j);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[j + e] += u[e];
        }
      }
    }
    if constexpr (SH > 1) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < V; ++j) sum[sh][l][j] = v[j];
      __syncthreads();
      if (sh > 0) continue;
#pragma unroll
      for (int k = 1; k < SH; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] += sum[k][l][j];
    }
    const float f = *out * (factor && p >= 0 ? factor[p] : 1.0f);
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] *= f;
    if (i < n) store16_f32(dx + (size_t)t * d + c, v);
  }
}

size_t up(size_t v) { return (v + 255) / 256 * 256; }

// Sizes of a call's tiles, pieces and workspace.
struct Plan {
  TileSize logits;     // of the logits' launches
  TileSize pair;       // of dx with dW
  int piece;           // columns of a piece of the backward, a multiple of 256
  int fwd_piece;       // and of the forward
  int split;           // parts of K of dx
  // bf16, up to 32 tokens: dz in two bf16 values, its rounding and what that leaves (16 bits together), as
  // two rows of dx's and dW's products, with x twice.  A rounding is off by 2^-8 at most, alike in a token's
  // whole row of products, and few tokens do not average it out (dW against 64 bits: 1.0 to 1.6 times a bf16
  // output's own rounding).  A k-step of 64 rows of dW holds both: 5 tokens of d = 768 take as long, 32 of 1024 4 %
  // and 24 of 2048 7 % longer, but 64 tokens of d = 2048 14 %, 128 30 %.
  bool two;
  // bf16, more tokens than that, each with a gradient g of its own: dz is left without g and with 1 in its
  // label's entry, q, the rest of which goes with g into the rows of x for dW (rounded once) and of dx (in
  // fp32).  In dz, which is rounded, g q is off alike in all products of the token that matter: dx by 1.45
  // times a bf16 output's own rounding (now 1.0), dW by 1.43 to 1.50 times it (now 1.41).
  bool fold;
  int parts;           // partials of a row of the forward: two of each tile of columns
};

constexpr size_t kDzBytes = (size_t)256 << 20;  // dz of a piece, at most (or of kPad columns)
constexpr int kPad = 256;

int tile_rows(TileSize t) { return t == TILE_256x256 ? 256 : t == TILE_32x64 ? 32 : 64; }
int tile_cols(TileSize t) { return t == TILE_256x256 ? 256 : t == TILE_64x128 ? 128 : 64; }

// fp32: six tiles of 64 x 128 per CU, or 32 x 64 ones (as the grouped GEMMs).
TileSize f32_tiles(double tiles) { return tiles >= 6.0 * num_cus() ? TILE_64x128 : TILE_32x64; }

// When the last of `cus` CUs ends that take na tiles of time a, then nb of time b <= a, each when it is free.
double ends(int cus, long na, double a, long nb, double b) {
  if (a < b) {
    std::swap(a, b);
    std::swap(na, nb);
  }
  const long q = na / cus, r = na % cus;
  const double base[2] = {q * a, (q + 1) * a};
  const long n[2] = {cus - r, r};
  double best = r ? base[1] : base[0];
  if (nb == 0) return best;
  // the earliest time at which all of nb fit: some CU ends at it
  const double least = std::max(best, (na * a + nb * b) / cus);
  double found = INFINITY;
  for (int i = 0; i < 2; ++i) {
    if (n[i] == 0) continue;
    for (long k = std::max(0L, (long)((least - base[i]) / b) - 1);; ++k) {
      const double t = base[i] + k * b;
      if (t < least) continue;
      if (t >= found) break;
      long fit = 0;
      for (int j = 0; j < 2; ++j)
        if (t >= base[j]) fit += n[j] * (long)((t - base[j]) / b + 1e-9);
      if (fit >= nb) {
        found = t;
        break;
      }
    }
  }
  return std::max(best, found);
}

// Estimate (us) of dx, in `split` parts, with dW in fp32: the tiles' k-steps of 32 and their ends on the CUs.
// Large tiles are taken where it is a tenth less for them, also with fewer of them than six a CU (400 tokens,
// d = 1024, 8000 words 138 us against 152, 787 of 640 on 15290 285 against 306, and where it is not, 1500 of
// 128 on 30000 226 against 215, 4000 of 512 on 5000 417 against 363).
double f32_pair_us(const GemmArgs& dx, const GemmArgs& dw, TileSize t, int split) {
  const double step = t == TILE_32x64 ? 0.33 : 1.05, end = t == TILE_32x64 ? 0.6 : 2.0;
  const long cols = ceil_div(dx.N, tile_cols(t));
  return ends(num_cus(), ceil_div(dx.cap, tile_rows(t)) * cols * split, ceil_div(dx.K, 32 * split) * step + end,
              ceil_div(dw.M, tile_rows(t)) * cols, ceil_div(dw.cap, 32) * step + end);
}

// Estimate (us) of the backward in 256 x 256 tiles, by pieces of `piece` columns and `split` parts of K of
// dx: rounds of the logits' tiles; the longest XCD of dx with dW, whose tiles are dealt by the XCD; the
// partial sums' and, where dz leaves the last-level cache, its own traffic.  On eleven heads of 1500 to
// 16000 tokens, each timed in 1 to 7 pieces by 1 to 6 parts, the pair that it picks is 0.4 % over the
// fastest; as few pieces as hold dz and dx in three quarters of the CUs 3.3 % (8192 tokens, d = 2048,
// 49152 words 3.91 ms against 4.06, 4096 tokens, d = 1024, 32000 words 704 us against 763).
double backward_us(const moe_xent& x, int width, int piece, int split) {
  const double step = 1.646, tile = 6.0;  // a 64-deep k-step; fill and epilogue
  const long rows = ceil_div(x.N, 256), cols = ceil_div(x.d, 256), words = piece / 256;
  const double logits = (double)((rows * words + num_cus() - 1) / num_cus()) * (x.d / 64 * 1.45 + 5.5);
  const double pair = ends(num_cus() / 8, (words * cols + 7) / 8, ceil_div(x.N, 64) * step + tile,
                           (rows * cols * split + 7) / 8, piece / 64.0 / split * step + tile);
  const double dz = 2.0 * x.N * piece, spill = dz > (double)(192 << 20) ? 0.9 * dz / 4.9e6 : 0.0;
  return ceil_div(width, piece) * (logits + pair + 9.6 * split * x.N * x.d / 4.9e6 + spill + 8.0);
}

Plan plan_of(const moe_xent& x, bool bwd) {
  const bool bf16 = x.dtype == MOE_BF16;
  const size_t s = bf16 ? 2 : 4;
  Plan p{};
  const int width = (int)up((size_t)x.V);
  // a piece's operands (rows of W and dW) below 2 GiB, its logits in 2^23 tiles of 32 x 64: a grid holds less
  // than 2^32 threads (a larger one is not refused but taken modulo 2^32)
  const size_t most_w =
      std::max<size_t>(kPad, std::min(((size_t)2 << 30) / ((size_t)x.d * 4),
                                      ((size_t)1 << 23) / (size_t)std::max(1, ceil_div(x.N, 32)) * 64) / kPad * kPad);
  p.fwd_piece = (int)std::min<size_t>(most_w, (size_t)width);
  GemmArgs z{}, dx{}, dw{};
  z.n_groups = dx.n_groups = dw.n_groups = 1;
  z.cap = dx.cap = dw.cap = x.N;
  z.N = std::min(x.V, p.fwd_piece); z.K = x.d;
  p.logits = bf16 ? xent_logit_tiles(z) : f32_tiles((double)ceil_div(x.N, 64) * ceil_div(z.N, 128));
  p.parts = ceil_div(x.V, tile_cols(p.logits)) * 2;  // (pieces are whole tiles)
  if (!bwd) return p;
  p.two = bf16 && x.N <= kTwo;
  if (p.two && p.logits == TILE_256x256) p.logits = TILE_64x128;  // (which write both)
  p.fold = bf16 && !p.two && x.dloss;
  dx.cap = dw.cap = p.two ? 2 * x.N : x.N;
  // Parts of K of dx: its few tiles reduce over the whole piece, so they are cut until they are three
  // quarters of the CUs (fp32, several of whose tiles share a CU: one and a half times them); 256 columns a
  // part at least.  Measured (us of the backward by parts): 512 tokens, d = 2048, 32768 words 1 698, 2 394, 4
  // 253, 8 212, 14 212, 28 242; 1531 tokens, d = 768, 50003 words 1055, 590, 365, 283, 284, 309; fp32, dx with
  // dW of 1000 tokens, d = 256, 30000 words 473 at three quarters, 279, and 281 at three times the CUs.
  const double most = (double)(((size_t)256 << 20) / ((size_t)std::max(1, dx.cap) * x.d * 4));
  auto split_of = [&](TileSize t) {
    const double tiles = (double)ceil_div(dx.cap, tile_rows(t)) * ceil_div(x.d, tile_cols(t));
    const double fill = (bf16 ? 0.75 : 1.5) * num_cus();
    return (int)std::max(1.0, std::min({fill / std::max(tiles, 1.0), p.piece / 256.0, most}));
  };
  const size_t most_dz = std::max<size_t>(kPad, kDzBytes / (std::max(1, x.N) * s) / kPad * kPad);
  const int pieces = (int)((width + std::min(most_w, most_dz) - 1) / std::min(most_w, most_dz));
  p.piece = (int)up((size_t)ceil_div(width, pieces));
  dx.N = x.d; dx.K = std::min(x.V, p.piece);
  dw.M = dx.K; dw.N = x.d;
  dw.xe.out_bf16 = x.dw_dtype == MOE_BF16;
  if (bf16) {
    const int split[3] = {split_of(TILE_256x256), split_of(TILE_64x128), split_of(TILE_64x64)};
    p.pair = xent_pair_tiles(dx, dw, split);
  } else {
    p.pair = f32_tiles((double)ceil_div(x.d, 128) * (ceil_div(x.N, 64) + ceil_div(dw.M, 64)));
    if (p.pair == TILE_32x64 && f32_pair_us(dx, dw, TILE_64x128, split_of(TILE_64x128)) <
                                    0.9 * f32_pair_us(dx, dw, TILE_32x64, split_of(TILE_32x64)))
      p.pair = TILE_64x128;
  }
  p.split = split_of(p.pair);
  if (p.pair != TILE_256x256 || p.logits != TILE_256x256) return p;
  const int whole = p.piece, few = p.split;  // (few tokens: more parts than eight)
  double least = backward_us(x, width, whole, few);
  for (int n = pieces; n < pieces + 5 && n <= width / kPad; ++n) {
    const int piece = (int)up((size_t)ceil_div(width, n));
    for (int split = 1; split <= 8 && split <= piece / 256 && split <= std::max(1.0, most); ++split) {
      const double us = backward_us(x, width, piece, split);
      if (us < least) {
        least = us;
        p.piece = piece;
        p.split = split;
      }
    }
  }
  return p;
}

struct Space {
  char* at;
  size_t used = 0;
  template <class T>
  T* take(size_t n) {
    T* p = at ? reinterpret_cast<T*>(at + used) : nullptr;
    used += up(n * sizeof(T));
    return p;
  }
};

struct Buffers {
  RowArgs row;
  float2* part;
  float* z_label;
  double* sums;
  int* done;
  void* dz;
  float* dx_part;
  size_t bytes;
};

// Tokens of a block of xent_loss.
int loss_rows(int N) { return N >= 8192 ? 32 : N >= 1024 ? 16 : 4; }

Buffers buffers(const moe_xent& x, const Plan& p, bool bwd, void* ws) {
  const size_t s = x.dtype == MOE_BF16 ? 2 : 4, N = x.N, M = p.two ? 2 * N : N;
  Space w{static_cast<char*>(ws)};
  Buffers b{};
  RowArgs& r = b.row;
  r.x = x.x; r.label = x.labels; r.N = x.N; r.d = x.d; r.V = x.V; r.size = (int)s; r.scale = x.scale;
  r.lse = x.lse; r.dloss = x.dloss;
  r.count = w.take<int>((N + kCountRows - 1) / kCountRows);
  r.pos = w.take<int>(N);
  r.off = w.take<int>(4);
  r.row_label = w.take<int>(N);
  r.two = p.two;
  r.xc = w.take<char>(M * x.d * s);
  if (!bwd) {
    b.z_label = w.take<float>(N);
    b.part = w.take<float2>((size_t)p.parts * N);
    b.sums = w.take<double>(2 * ((N + loss_rows(x.N) - 1) / loss_rows(x.N)));
    b.done = w.take<int>(1);
  } else {
    r.row_lse = w.take<float>(N);
    r.coef = w.take<float>(N);
    r.out = w.take<float>(1);
    if (x.dtype == MOE_BF16 && !p.two) {  // (whether dloss is given or not: sizes do not depend on it)
      r.xs = w.take<char>(N * x.d * s);
      r.factor = w.take<float>(N);
    }
    r.fold = p.fold; r.w = x.w; r.z2 = 2.0f * x.z_coef;
    b.dz = w.take<char>(M * p.piece * s);
    b.dx_part = w.take<float>((size_t)p.split * M * x.d);
    r.n_counters = ceil_div(x.V, p.piece) * kXcdCounters;
    r.counters = w.take<int>(r.n_counters);
  }
  b.bytes = w.used;
  return b;
}

template <bool BWD>
hipError_t rows(const Buffers& b, hipStream_t s) {
  const RowArgs& r = b.row;
  if (r.N > kDirect) {
    MOE_TIMED("xent_count", s,
              xent_count_kernel<<<ceil_div(r.N, kCountRows), 256, 0, s>>>(r.label, r.N, r.count));
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  if (r.N <= 4096) MOE_TIMED("xent_rows", s, xent_rows_kernel<BWD, 4><<<ceil_div(r.N, 4), 256, 0, s>>>(r));
  else MOE_TIMED("xent_rows", s, xent_rows_kernel<BWD, 16><<<ceil_div(r.N, 16), 256, 0, s>>>(r));
  return hipGetLastError();
}

// The logits' product of columns [v0, v0 + V): operands and what its epilogue takes.
GemmArgs logits(const moe_xent& x, const Buffers& b, int v0, int V) {
  const size_t s = x.dtype == MOE_BF16 ? 2 : 4;
  GemmArgs a{};
  a.offsets = b.row.off; a.n_groups = 1; a.cap = x.N;
  a.A = b.row.xc; a.lda = x.d;
  a.B = static_cast<const char*>(x.w) + (size_t)v0 * x.d * s; a.ldb = x.d;
  a.N = V; a.K = x.d;
  a.xe.x_all = x.x;
  a.xe.label = b.row.row_label;
  a.xe.lse = b.row.row_lse;
  a.xe.coef = b.row.coef;
  a.xe.out = b.row.out;
  a.xe.V = V; a.xe.v0 = v0;
  a.xe.scale = x.scale; a.xe.z2 = 2.0f * x.z_coef;
  return a;
}

hipError_t run(TileSize size, int bf16, int ka, const GemmArgs& a, const GemmArgs* b, int* counters,
               hipStream_t s) {
  if (size == TILE_256x256) return run_gemm_xent(ka, a, b, counters, s);
  return run_gemm_tile(bf16, ka, b ? XE_DW : ka, &a, 1, b, b ? 1 : 0, size, s);
}

}  // namespace

size_t xent_fwd_ws_bytes(const moe_xent* x) { return buffers(*x, plan_of(*x, false), false, nullptr).bytes; }
size_t xent_bwd_ws_bytes(const moe_xent* x) { return buffers(*x, plan_of(*x, true), true, nullptr).bytes; }

hipError_t launch_xent_fwd(const moe_xent* x, hipStream_t s) {
  const Plan p = plan_of(*x, false);
  const int bf16 = x->dtype == MOE_BF16;
  const Buffers b = buffers(*x, p, false, x->ws);
  hipError_t e;
  if (x->N == 0) {
    MOE_TIMED("xent_none", s, xent_none_kernel<<<1, 64, 0, s>>>(x->total));
    return hipGetLastError();
  }
  // Few tokens: every row as it is (rows are independent here).  In bf16 leaving some out saves no tile of 256 and
  // little of W's stream, less than its launch takes: 24 tokens 55 -> 51 us, 256 of d = 2048 on 49152 words 59 ->
  // 55, half of them left out 57 -> 54.  In fp32 that holds of small heads (256 of d = 64 on 1000 words 14 -> 11 us,
  // 512 on 8000 32 -> 29) and of tokens that all count (256 of 2048 on 49152 388 -> 384); the products bound
  // large ones, whose left-out tokens cost what others do (half of those 256: 384 us, and 210 without them).
  const bool as_is = x->N <= kFew;
  if (!as_is && (e = rows<false>(b, s)) != hipSuccess) return e;
  const int width = tile_cols(p.logits) / 2;  // of a partial: half a tile's columns
  int parts = 0;
  for (int v0 = 0; v0 < x->V; v0 += p.fwd_piece) {
    const int V = std::min(x->V - v0, p.fwd_piece);
    GemmArgs a = logits(*x, b, v0, V);
    a.xe.part = b.part + (size_t)parts * x->N;
    a.xe.z_label = b.z_label;
    a.xe.done = b.done;
    if (as_is) {
      a.offsets = nullptr;
      a.xe.label = x->labels;
    }
    if ((e = run(p.logits, bf16, XE_LSE, a, nullptr, nullptr, s)) != hipSuccess) return e;
    parts += ceil_div(V, 2 * width) * 2;
  }
  const int R = loss_rows(x->N), blocks = ceil_div(x->N, R);
#define XENT_LOSS(R_)                                                                                    \
  MOE_TIMED("xent_loss", s,                                                                              \
            xent_loss_kernel<R_><<<blocks, kLossThreads, 0, s>>>(                                        \
                x->N, x->V, parts, x->z_coef, x->labels, as_is ? nullptr : b.row.pos, b.part, b.z_label, \
                x->loss, x->lse, b.sums, b.done, x->total))
  if (R == 32) XENT_LOSS(32);
  else if (R == 16) XENT_LOSS(16);
  else XENT_LOSS(4);
#undef XENT_LOSS
  return hipGetLastError();
}

hipError_t launch_xent_bwd(const moe_xent* x, hipStream_t s) {
  const Plan p = plan_of(*x, true);
  const int bf16 = x->dtype == MOE_BF16;
  const size_t es = bf16 ? 2 : 4, ws = x->dw_dtype == MOE_BF16 ? 2 : 4;
  const Buffers b = buffers(*x, p, true, x->ws);
  hipError_t e;
  if (x->N > 0 && (e = rows<true>(b, s)) != hipSuccess) return e;
  for (int v0 = 0; x->N > 0 && v0 < x->V; v0 += p.piece) {
    const int V = std::min(x->V - v0, p.piece), ld = (int)up((size_t)V);
    GemmArgs a = logits(*x, b, v0, V);
    a.C = b.dz; a.ldc = ld;
    a.N = ld;  // (the columns past V are written too: zeros)
    if (p.two) {
      a.ldc = 2L * ld; a.xe.lo = ld;
      a.lda = 2L * x->d; a.xe.x_all = b.row.xc;
    }
    if ((e = run(p.logits, bf16, XE_DZ, a, nullptr, nullptr, s)) != hipSuccess) return e;
    GemmArgs dx = a, dw = a;
    if (p.two) {
      dx.offsets = dw.offsets = b.row.off + 2;
      dx.cap = dw.cap = 2 * x->N;
    }
    dx.A = b.dz; dx.lda = ld;
    dx.N = x->d; dx.K = p.pair == TILE_256x256 ? ld : V;
    dx.part = b.dx_part; dx.c_split = (long)dx.cap * x->d; dx.ksplit = p.split;
    dx.accumulate = v0 > 0;
    dw.A = b.dz; dw.lda = ld;
    dw.B = b.row.xc; dw.ldb = x->d;
    if (p.fold) dw.B = dw.xe.x_all = b.row.xs;
    dw.C = static_cast<char*>(x->dw) + (size_t)v0 * x->d * ws; dw.ldc = x->d;
    dw.M = ld; dw.N = x->d;
    dw.accumulate = x->accumulate_dw;
    dw.xe.out_bf16 = x->dw_dtype == MOE_BF16;
    if ((e = run(p.pair, bf16, XE_DX, dx, &dw, b.row.counters + v0 / p.piece * kXcdCounters, s)) != hipSuccess)
      return e;
  }
  if (x->N == 0) {
    const size_t n = (size_t)x->V * x->d * ws / 16;
    if (!x->accumulate_dw)
      MOE_TIMED("xent_clear", s, xent_clear_kernel<<<(int)std::min<size_t>(2048, (n + 255) / 256), 256, 0, s>>>(
          static_cast<u32x4_t*>(x->dw), n));
    return hipGetLastError();
  }
  const size_t n = (size_t)x->N * x->d / (bf16 ? 8 : 4);
  const bool share = p.two || (p.split >= 8 && n < (size_t)num_cus() * 256);
  const int blocks = (int)std::min<size_t>(8192, share ? (n + 31) / 32 : (n + 255) / 256);
  const size_t stride = (size_t)x->N * x->d * (p.two ? 2 : 1);
#define XENT_DX(E_, SH_, TWO_)                                                 \
  MOE_TIMED("xent_dx", s, xent_dx_kernel<E_, SH_, TWO_><<<blocks, 256, 0, s>>>( \
      static_cast<E_*>(x->dx), b.row.pos, b.dx_part, stride, p.split, x->N, x->d, b.row.out, \
      p.fold ? b.row.factor : nullptr))
  if (p.two) XENT_DX(bf16_t, 8, true);
  else if (bf16 && share) XENT_DX(bf16_t, 8, false);
  else if (bf16) XENT_DX(bf16_t, 1, false);
  else if (share) XENT_DX(float, 8, false);
  else XENT_DX(float, 1, false);
#undef XENT_DX
  return hipGetLastError();
}

}  // namespace moe
