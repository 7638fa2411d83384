// The norm of many gradients together, and clipping by it.
//
//   norm = sqrt(sum over all tensors of g^2);  scale = norm > max_norm ? max_norm / norm : 1
//   out = scale g, rounded once
//
// Bound by HBM: the norm reads every value once, clipping reads and writes it once more (AdamW
// with the scale, optim.hip, saves that).  Sums are held in fp64: squares of fp32 values neither
// overflow nor vanish there, and the conversions and multiply-adds take a fraction of the loads'
// time.
//
// A launch covers many tensors (GradTable), whose table is a kernel argument: no list is copied to
// the device, and a captured launch keeps its own.  Tensors are cut into chunks (chunk_of),
// which the blocks take in turn; every block stores one partial sum, and a last block adds the
// partials of all launches in order, so the result does not depend on timing.
//
// Measured: four tensors of 2^26 fp32 values, norm 183 us (5.9 TB/s), with clipping to other tensors 625 (5.2
// TB/s); 300 of 2^14 values 15 and 27 us; one of 4096 values 9 and 15 us, two and three launches' latency.
#include <cmath>

#include "common.h"
#include "kernels.h"
#include "timing.h"

namespace moe {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxChunk = 16384;
constexpr int kMostChunks = 1 << 30;  // of a launch: those of the largest tensor

// Tensors of a launch: their pointers, the chunks before each, and the values of each one's last
// chunk less one, with the type in the top bit (14 or 22 bytes a tensor, so that a launch takes as
// many as it can).
template <int N, bool OUT>
struct GradTable {
  static constexpr int kTensors = N;
  const void* p[N];
  void* out[OUT ? N : 1];
  int first[N + 1];
  uint16_t tail[N];
  int count, chunk;
};
typedef GradTable<272, false> NormTable;
typedef GradTable<174, true> ClipTable;
static_assert(sizeof(NormTable) <= 3968 && sizeof(ClipTable) <= 3968, "kernel arguments hold 4 KiB");
static_assert(kMaxChunk <= 32768, "a tail has 15 bits");

// The tensor of chunk c (wave-uniform).
template <class T>
DEVI int tensor_of(const T& t, int c) {
  int lo = 0, hi = t.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= c) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// Chunk c of a table: its tensor, where it starts there, its values and their type.
struct Chunk {
  int q;
  size_t at, n;
  bool bf16;
};
template <class T>
DEVI Chunk chunk_at(const T& t, int c) {
  Chunk k;
  k.q = tensor_of(t, c);
  k.at = (size_t)(c - t.first[k.q]) * t.chunk;
  const unsigned tail = t.tail[k.q];
  k.n = c + 1 < t.first[k.q + 1] ? (size_t)t.chunk : (tail & 0x7fff) + 1;
  k.bf16 = tail >> 15;
  return k;
}

// The sum of the squares of n values at p, in the block's threads.
template <class E>
DEVI double square_sum(const E* p, size_t n) {
  constexpr int V = Vec16<E>::N;
  double s = 0.0;
  if ((reinterpret_cast<uintptr_t>(p) & 15u) == 0) {
    const int nv = (int)(n / V);
#pragma unroll 4
    for (int i = threadIdx.x; i < nv; i += kThreads) {
      float v[V];
      load16_f32(p + (size_t)i * V, v);
#pragma unroll
      for (int j = 0; j < V; ++j) s += (double)v[j] * (double)v[j];
    }
    for (size_t i = (size_t)nv * V + threadIdx.x; i < n; i += kThreads) {
      const double v = (double)to_f32(p[i]);
      s += v * v;
    }
  } else {
    for (size_t i = threadIdx.x; i < n; i += kThreads) {
      const double v = (double)to_f32(p[i]);
      s += v * v;
    }
  }
  return s;
}

DEVI double wave_sum_f64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

__global__ __launch_bounds__(kThreads) void grad_norm_kernel(NormTable t, double* part) {
  __shared__ double sum[kThreads / 64];
  const int chunks = t.first[t.count];
  double s = 0.0;
  for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
    const Chunk k = chunk_at(t, c);
    s += k.bf16 ? square_sum(static_cast<const bf16_t*>(t.p[k.q]) + k.at, k.n)
                : square_sum(static_cast<const float*>(t.p[k.q]) + k.at, k.n);
  }
  s = wave_sum_f64(s);
  if ((threadIdx.x & 63) == 0) sum[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) s += sum[w];
    part[blockIdx.x] = s;
  }
}

// norm[0], norm[1] = the norm and the scale, from n partial sums.  A norm that is not finite has
// the scale NaN.
__global__ __launch_bounds__(1024) void grad_norm_sum_kernel(const double* part, int n, float max_norm,
                                                             float* norm) {
  __shared__ double sum[16];
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += 1024) s += part[i];
  s = wave_sum_f64(s);
  if ((threadIdx.x & 63) == 0) sum[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < 16; ++w) s += sum[w];
    const float v = (float)sqrt(s);
    norm[0] = v;
    norm[1] = !(v < INFINITY) ? NAN : v > max_norm ? max_norm / v : 1.0f;
  }
}

template <class E>
DEVI void scale_to(const E* p, E* out, size_t n, float scale) {
  constexpr int V = Vec16<E>::N;
  size_t done = 0;
  if (((reinterpret_cast<uintptr_t>(p) | reinterpret_cast<uintptr_t>(out)) & 15u) == 0) {
    const int nv = (int)(n / V);
#pragma unroll 4
    for (int i = threadIdx.x; i < nv; i += kThreads) {
      float v[V];
      load16_f32(p + (size_t)i * V, v);
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] *= scale;
      store16_f32(out + (size_t)i * V, v);
    }
    done = (size_t)nv * V;
  }
  for (size_t i = done + threadIdx.x; i < n; i += kThreads) out[i] = from_f32<E>(to_f32(p[i]) * scale);
}

__global__ __launch_bounds__(kThreads) void grad_clip_kernel(ClipTable t, const float* norm) {
  // (scale 1, or NaN: nothing to clip, so that values in place stay as they are)
  const float s = norm[1], scale = s < 1.0f ? s : 1.0f;
  const int chunks = t.first[t.count];
  for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
    const Chunk k = chunk_at(t, c);
    const void* const p = t.p[k.q];
    void* const out = t.out[k.q];
    if (scale == 1.0f && p == out) continue;
    if (k.bf16)
      scale_to(static_cast<const bf16_t*>(p) + k.at, static_cast<bf16_t*>(out) + k.at, k.n, scale);
    else
      scale_to(static_cast<const float*>(p) + k.at, static_cast<float*>(out) + k.at, k.n, scale);
  }
}

// Values of a chunk, multiples of what 256 threads load at once: large ones cost a block's search and its
// first load's latency less often, small ones spread a list over more blocks (300 tensors of 64 to 2^17
// values clipped: 10 us less in chunks of 4096 than of 16384).
int chunk_of(const moe_grad* g, int n) {
  size_t total = 0;
  for (int i = 0; i < n; ++i) total += g[i].n;
  return total < ((size_t)32 << 20) ? 4096 : kMaxChunk;
}

// Blocks of a launch of `chunks` chunks: all that are resident at once, 8 of 256 threads a CU.
int chunk_blocks(int chunks) { return std::min(chunks, 8 * num_cus()); }

// f(table, blocks) for launches of up to T::kTensors tensors with values.
template <class T, class F>
hipError_t for_tables(const moe_grad* g, int n, F&& f) {
  T t;
  t.chunk = chunk_of(g, n);
  t.count = 0;
  t.first[0] = 0;
  for (int i = 0; i <= n; ++i) {
    const bool end = i == n;
    // (a launch's chunks, and a block's steps past the last of them, are counted in 31 bits: a tensor that
    // does not fit opens the next)
    const int64_t chunks = end ? 0 : (int64_t)((g[i].n + t.chunk - 1) / t.chunk);
    if (t.count > 0 && (end || t.count == T::kTensors || t.first[t.count] + chunks > kMostChunks)) {
      if (const hipError_t e = f(t, chunk_blocks(t.first[t.count])); e != hipSuccess) return e;
      t.count = 0;
    }
    if (end || chunks == 0) continue;
    t.p[t.count] = g[i].grad;
    if constexpr (sizeof(t.out) > sizeof(void*)) t.out[t.count] = g[i].out;
    t.tail[t.count] = (uint16_t)((g[i].n - 1) % t.chunk | (g[i].dtype == MOE_BF16 ? 0x8000 : 0));
    t.first[t.count + 1] = t.first[t.count] + (int)chunks;
    ++t.count;
  }
  return hipSuccess;
}

}  // namespace

size_t grad_norm_ws_bytes(const moe_grad* g, int n) {
  size_t parts = 0;
  (void)for_tables<NormTable>(g, n, [&](const NormTable&, int blocks) {
    parts += blocks;
    return hipSuccess;
  });
  return parts * sizeof(double);
}

hipError_t launch_grad_norm(const moe_grad* g, int n, float max_norm, float* norm, void* ws,
                            hipStream_t s) {
  double* const part = static_cast<double*>(ws);
  int parts = 0;
  const hipError_t e = for_tables<NormTable>(g, n, [&](const NormTable& t, int blocks) {
    MOE_TIMED("grad_norm", s, grad_norm_kernel<<<blocks, kThreads, 0, s>>>(t, part + parts));
    parts += blocks;
    return hipGetLastError();
  });
  if (e != hipSuccess) return e;
  MOE_TIMED("grad_norm_sum", s, grad_norm_sum_kernel<<<1, 1024, 0, s>>>(part, parts, max_norm, norm));
  return hipGetLastError();
}

hipError_t launch_grad_clip(const moe_grad* g, int n, const float* norm, hipStream_t s) {
  return for_tables<ClipTable>(g, n, [&](const ClipTable& t, int blocks) {
    MOE_TIMED("grad_clip", s, grad_clip_kernel<<<blocks, kThreads, 0, s>>>(t, norm));
    return hipGetLastError();
  });
}

}  // namespace moe
