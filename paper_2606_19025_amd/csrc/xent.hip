// Softmax cross entropy of a linear head over a vocabulary, without keeping the logits.
//
//   z_tv = scale x_t . w_v;   lse_t = log sum_v exp z_tv;   loss_t = lse_t - z_ty + z_coef lse_t^2
//   dz_tv = g_t ((1 + 2 z_coef lse_t) exp(z_tv - lse_t) - [v = y_t])
//   dx = scale dz W,  dW = scale dz^T x            (the scale goes into g_t)
//
// Four products of 2 N V d operations (gemm.hip, gemm_tile.hip: XE_* kinds).  Forward: a tile of
// logits ends in (max, sum of 2^(z - max)) of each of its rows, and the label's logit where it is
// among its columns; a second launch joins the pieces of a row.  Backward, for one piece of the
// vocabulary after the other: the logits again, which end as dz in dtype, then dx and dW of the
// piece in one launch.  dx is summed over pieces (and parts of K) in fp32 and rounded once.
//
// Tokens that do not count (label < 0) are left out of every product: the others' rows are copied
// together first (where all count, x itself is read), so a padded batch costs what its tokens
// do, and nothing that stands in a padded row enters a gradient.  How many there are stays on the
// device, as in the dispatch.
#include <algorithm>
#include <cmath>

#include "gemm.h"
#include "kernels.h"
#include "timing.h"

namespace moe {
namespace {

constexpr int kRows = 64;        // tokens of a block of the row kernels
constexpr int kCountRows = 1024; // tokens of a counting block
constexpr int kDirect = 8192;    // up to here every block counts all labels itself
constexpr int kSegments = 16;    // threads of a row of partials

struct RowArgs {
  const void* x;
  const int32_t* label;
  const float* lse;    // backward
  const float* dloss;  // backward, or NULL: 1 / the number of tokens that count
  int N, d, V, size;   // size: bytes of an element
  float scale;
  int* count;          // [blocks of kCountRows]
  int* pos;            // [N] row of a token among those that count, or -1
  int* off;            // {0, tokens that count}
  int* row_label;      // the rest by row
  float* z_label;      // forward
  float* row_lse;      // backward
  float* coef;
  void* xc;
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

// The rows of the tokens that count, kRows tokens a block.
template <bool BWD>
__global__ __launch_bounds__(256) void xent_rows_kernel(RowArgs a) {
  __shared__ int buf[4];
  __shared__ int row[kRows];
  const int t0 = blockIdx.x * kRows;
  // tokens that count before this block's, and all of them
  int before = 0, total = 0;
  if (a.N <= kDirect) {
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
    const int y = t < a.N ? a.label[t] : -1;
    const unsigned long long counts = __ballot(y >= 0);
    const int p = y < 0 ? -1 : before + __builtin_popcountll(counts & ((1ull << threadIdx.x) - 1));
    row[threadIdx.x] = p;
    if (t < a.N) a.pos[t] = p;
    if (p >= 0) {
      const bool in = y < a.V;
      a.row_label[p] = y;
      if constexpr (BWD) {
        a.row_lse[p] = a.lse[t];
        // (a label that is no word of the vocabulary makes what it enters NaN)
        a.coef[p] = in ? a.scale * (a.dloss ? a.dloss[t] : 1.0f / (float)total) : NAN;
      } else if (!in) {
        a.z_label[p] = NAN;
      }
    }
    if (blockIdx.x == 0 && threadIdx.x < 2) a.off[threadIdx.x] = threadIdx.x ? total : 0;
  }
  if (total == a.N) return;  // x itself is read
  __syncthreads();
  const int chunks = a.d * a.size / 16;
  const u32x4_t* src = static_cast<const u32x4_t*>(a.x);
  u32x4_t* dst = static_cast<u32x4_t*>(a.xc);
  for (int r = threadIdx.x >> 6; r < kRows; r += 4) {
    const int p = row[r];
    if (p < 0) continue;
    for (int c = threadIdx.x & 63; c < chunks; c += 64)
      dst[(size_t)p * chunks + c] = src[(size_t)(t0 + r) * chunks + c];
  }
}

// (max, sum) pairs of base 2 joined.
DEVI float2 join(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x);
  if (m == -INFINITY) return a;
  return float2{m, a.y * __builtin_amdgcn_exp2f(a.x - m) + b.y * __builtin_amdgcn_exp2f(b.x - m)};
}

// lse and loss of kRows tokens a block from their P partials; the block's sum of losses.
__global__ __launch_bounds__(kRows * kSegments) void xent_loss_kernel(
    int N, int P, float z_coef, const int* pos, const int* off, const float2* part, const float* z_label,
    float* loss, float* lse, double* sums, float* total) {
  __shared__ float2 seg[kSegments][kRows];
  const int r = threadIdx.x & (kRows - 1), q = threadIdx.x / kRows;
  const int t = blockIdx.x * kRows + r;
  const int p = t < N ? pos[t] : -1;
  float2 v = {-INFINITY, 0.f};
  if (p >= 0)
    for (int i = q; i < P; i += kSegments) v = join(v, part[(size_t)i * N + p]);
  seg[q][r] = v;
  __syncthreads();
  if (q != 0) return;
  float l = 0.f, out = 0.f;
  if (p >= 0) {
#pragma unroll
    for (int i = 1; i < kSegments; ++i) v = join(v, seg[i][r]);
    l = v.x * kLn2 + logf(v.y);
    out = l - z_label[p] + z_coef * l * l;
  }
  if (t < N) {
    lse[t] = l;
    loss[t] = out;
  }
  double s = (double)out;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if (r == 0) {
    if (gridDim.x > 1) {
      sums[blockIdx.x] = s;
    } else {
      total[0] = (float)s;
      total[1] = N > 0 ? (float)off[1] : 0.f;
    }
  }
}

__global__ __launch_bounds__(256) void xent_total_kernel(const double* sums, int n, const int* off,
                                                         float* total) {
  __shared__ double buf[4];
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += 256) s += sums[i];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    total[0] = (float)(buf[0] + buf[1] + buf[2] + buf[3]);
    total[1] = (float)off[1];
  }
}

__global__ __launch_bounds__(64) void xent_zero_kernel(int* counters, int n) {
  if ((int)threadIdx.x < n) counters[threadIdx.x] = 0;
}

// n 16-byte pieces of zeros (the gradient of no tokens).
__global__ __launch_bounds__(256) void xent_clear_kernel(u32x4_t* p, size_t n) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256)
    p[i] = u32x4_t{0u, 0u, 0u, 0u};
}

// dx[t] = the sum of its row's S partial sums in order, or zeros.
template <class E>
__global__ __launch_bounds__(256) void xent_dx_kernel(E* dx, const int* pos, const float* part, size_t stride,
                                                      int S, int N, int d) {
  constexpr int V = Vec16<E>::N;
  const int chunks = d / V;
  const size_t n = (size_t)N * chunks;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) {
    const int t = (int)(i / chunks), c = (int)(i % chunks) * V;
    const int p = pos[t];
    float v[V] = {};
    if (p >= 0)
      for (int s = 0; s < S; ++s) {
        const float* q = part + (size_t)s * stride + (size_t)p * d + c;
#pragma unroll
        for (int j = 0; j < V; j += 4) {
          const f32x4_t u = *reinterpret_cast<const f32x4_t*>(q + j);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[j + e] += u[e];
        }
      }
    store16_f32(dx + (size_t)t * d + c, v);
  }
}

size_t up(size_t v) { return (v + 255) / 256 * 256; }

// Sizes of a call's tiles, pieces and workspace.
struct Plan {
  bool large;          // 256 x 256 tiles
  TileSize tile;       // else
  int piece;           // columns of a piece of the backward, a multiple of 256
  int fwd_piece;       // and of the forward
  int split;           // parts of K of dx
  int parts;           // partials of a row (upper bound over the tile sizes)
};

constexpr size_t kDzBytes = (size_t)512 << 20;
constexpr int kPad = 256;

Plan plan_of(const moe_xent& x) {
  const bool bf16 = x.dtype == MOE_BF16;
  const size_t s = bf16 ? 2 : 4;
  Plan p{};
  p.large = bf16 && x.N > 128;
  if (bf16) p.tile = x.N <= 32 ? TILE_32x64 : TILE_64x128;
  else p.tile = (long)ceil_div(x.N, 64) * ceil_div(x.V, 128) >= 6L * num_cus() ? TILE_64x128 : TILE_32x64;
  const int width = up((size_t)x.V);
  // a piece's operands (rows of W and dW) below 2 GiB, dz within its budget
  const size_t most_w = std::max<size_t>(kPad, ((size_t)2 << 30) / ((size_t)x.d * 4) / kPad * kPad);
  const size_t most_dz = std::max<size_t>(kPad, kDzBytes / (std::max(1, x.N) * s) / kPad * kPad);
  const int pieces = (int)((width + std::min(most_w, most_dz) - 1) / std::min(most_w, most_dz));
  p.piece = (int)up((size_t)ceil_div(width, pieces));
  p.fwd_piece = (int)std::min<size_t>(most_w, (size_t)width);
  p.parts = ceil_div(x.V, 64) * 2 + 2;
  // parts of K of dx, so that its few long tiles take no longer than all tiles by CUs
  const int bm = p.large ? 256 : p.tile == TILE_32x64 && !bf16 ? 32 : 64, bn = p.large ? 256 : bm * 2;
  const double dx_tiles = (double)ceil_div(x.N, bm) * ceil_div(x.d, bn);
  const double dw_tiles = (double)ceil_div(p.piece, bm) * ceil_div(x.d, bn);
  const int slots = num_cus() * (p.large ? 1 : 4);
  const double share = std::max((dx_tiles * p.piece + dw_tiles * x.N) / slots, 512.0);
  const size_t most = ((size_t)256 << 20) / ((size_t)std::max(1, x.N) * x.d * 4);
  p.split = (int)std::max<double>(1, std::min<double>({p.piece / share, 32.0, (double)most}));
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
  double* sums;
  void* dz;
  float* dx_part;
  int* counters;
  size_t bytes;
};

Buffers buffers(const moe_xent& x, const Plan& p, bool bwd, void* ws) {
  const size_t s = x.dtype == MOE_BF16 ? 2 : 4, N = x.N;
  Space w{static_cast<char*>(ws)};
  Buffers b{};
  RowArgs& r = b.row;
  r.x = x.x; r.label = x.labels; r.N = x.N; r.d = x.d; r.V = x.V; r.size = (int)s; r.scale = x.scale;
  r.lse = x.lse; r.dloss = x.dloss;
  r.count = w.take<int>((N + kCountRows - 1) / kCountRows);
  r.pos = w.take<int>(N);
  r.off = w.take<int>(2);
  r.row_label = w.take<int>(N);
  r.xc = w.take<char>(N * x.d * s);
  if (!bwd) {
    r.z_label = w.take<float>(N);
    b.part = w.take<float2>((size_t)p.parts * N);
    b.sums = w.take<double>((N + kRows - 1) / kRows);
  } else {
    r.row_lse = w.take<float>(N);
    r.coef = w.take<float>(N);
    b.dz = w.take<char>(N * p.piece * s);
    b.dx_part = w.take<float>((size_t)p.split * N * x.d);
    b.counters = w.take<int>(64);
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
  MOE_TIMED("xent_rows", s, xent_rows_kernel<BWD><<<ceil_div(r.N, kRows), 256, 0, s>>>(r));
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
  a.xe.V = V; a.xe.v0 = v0;
  a.xe.scale = x.scale; a.xe.z2 = 2.0f * x.z_coef;
  return a;
}

hipError_t run(const Plan& p, int bf16, int ka, const GemmArgs& a, const GemmArgs* b, int* counters,
               hipStream_t s) {
  if (p.large) return run_gemm_xent(ka, a, b, counters, s);
  const TileSize size = b && p.tile == TILE_32x64 ? TILE_64x128 : p.tile;
  return run_gemm_tile(bf16, ka, b ? XE_DW : ka, &a, 1, b, b ? 1 : 0, size, s);
}

}  // namespace

size_t xent_fwd_ws_bytes(const moe_xent* x) { return buffers(*x, plan_of(*x), false, nullptr).bytes; }
size_t xent_bwd_ws_bytes(const moe_xent* x) { return buffers(*x, plan_of(*x), true, nullptr).bytes; }

hipError_t launch_xent_fwd(const moe_xent* x, hipStream_t s) {
  const Plan p = plan_of(*x);
  const int bf16 = x->dtype == MOE_BF16;
  const Buffers b = buffers(*x, p, false, x->ws);
  hipError_t e;
  if (x->N > 0 && (e = rows<false>(b, s)) != hipSuccess) return e;
  const int width = p.large ? 128 : p.tile == TILE_32x64 ? 32 : 64;  // of a partial: half a tile's columns
  int parts = 0;
  for (int v0 = 0; x->N > 0 && v0 < x->V; v0 += p.fwd_piece) {
    const int V = std::min(x->V - v0, p.fwd_piece);
    GemmArgs a = logits(*x, b, v0, V);
    a.xe.part = b.part + (size_t)parts * x->N;
    a.xe.z_label = b.row.z_label;
    if ((e = run(p, bf16, XE_LSE, a, nullptr, nullptr, s)) != hipSuccess) return e;
    parts += ceil_div(V, 2 * width) * 2;
  }
  const int blocks = std::max(1, ceil_div(x->N, kRows));
  MOE_TIMED("xent_loss", s,
            xent_loss_kernel<<<blocks, kRows * kSegments, 0, s>>>(
                x->N, parts, x->z_coef, b.row.pos, b.row.off, b.part, b.row.z_label, x->loss, x->lse,
                b.sums, x->total));
  if ((e = hipGetLastError()) != hipSuccess || blocks == 1) return e;
  MOE_TIMED("xent_total", s, xent_total_kernel<<<1, 256, 0, s>>>(b.sums, blocks, b.row.off, x->total));
  return hipGetLastError();
}

hipError_t launch_xent_bwd(const moe_xent* x, hipStream_t s) {
  const Plan p = plan_of(*x);
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
    if ((e = run(p, bf16, XE_DZ, a, nullptr, nullptr, s)) != hipSuccess) return e;
    GemmArgs dx = a, dw = a;
    dx.A = b.dz; dx.lda = ld;
    dx.N = x->d; dx.K = p.large ? ld : V;
    dx.part = b.dx_part; dx.c_split = (long)x->N * x->d; dx.ksplit = p.split;
    dx.accumulate = v0 > 0;
    dw.A = b.dz; dw.lda = ld;
    dw.B = b.row.xc; dw.ldb = x->d;
    dw.C = static_cast<char*>(x->dw) + (size_t)v0 * x->d * ws; dw.ldc = x->d;
    dw.M = ld; dw.N = x->d;
    dw.accumulate = x->accumulate_dw;
    dw.xe.out_bf16 = x->dw_dtype == MOE_BF16;
    if (p.large) {
      MOE_TIMED("xent_zero", s, xent_zero_kernel<<<1, 64, 0, s>>>(b.counters, kXcdCounters));
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if ((e = run(p, bf16, XE_DX, dx, &dw, b.counters, s)) != hipSuccess) return e;
  }
  if (x->N == 0) {
    const size_t n = (size_t)x->V * x->d * ws / 16;
    if (!x->accumulate_dw)
      MOE_TIMED("xent_clear", s, xent_clear_kernel<<<(int)std::min<size_t>(2048, (n + 255) / 256), 256, 0, s>>>(
          static_cast<u32x4_t*>(x->dw), n));
    return hipGetLastError();
  }
  const size_t n = (size_t)x->N * x->d / (bf16 ? 8 : 4);
  const int blocks = (int)std::min<size_t>(8192, (n + 255) / 256);
  if (bf16)
    MOE_TIMED("xent_dx", s, xent_dx_kernel<bf16_t><<<blocks, 256, 0, s>>>(
        static_cast<bf16_t*>(x->dx), b.row.pos, b.dx_part, (size_t)x->N * x->d, p.split, x->N, x->d));
  else
    MOE_TIMED("xent_dx", s, xent_dx_kernel<float><<<blocks, 256, 0, s>>>(
        static_cast<float*>(x->dx), b.row.pos, b.dx_part, (size_t)x->N * x->d, p.split, x->N, x->d));
  return hipGetLastError();
}

}  // namespace moe
