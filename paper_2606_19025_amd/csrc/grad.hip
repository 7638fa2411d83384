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
// A launch covers up to kTensors tensors, whose table is a kernel argument: no list is copied to
// the device, and a captured launch keeps its own.  Tensors are cut into chunks (chunk_of),
// which the blocks take in turn; every block stores one partial sum, and a last block adds the
// partials of all launches in order, so the result does not depend on timing.
#include <cmath>

#include "common.h"
#include "kernels.h"
#include "timing.h"

namespace moe {
namespace {

constexpr int kTensors = 112;
constexpr int kThreads = 256;

struct GradTable {
  const void* p[kTensors];
  void* out[kTensors];
  size_t n[kTensors];
  int first[kTensors + 1];  // chunks before each tensor
  uint8_t bf16[kTensors];
  int count, chunk;
};
static_assert(sizeof(GradTable) <= 3900, "kernel arguments hold 4 KiB");

// The tensor of chunk c (wave-uniform).
DEVI int tensor_of(const GradTable& t, int c) {
  int lo = 0, hi = t.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= c) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// f(i, v, N) for the values of [begin, end) in vectors of 16 bytes (VEC) or one by one.
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

__global__ __launch_bounds__(kThreads) void grad_norm_kernel(GradTable t, double* part) {
  __shared__ double sum[kThreads / 64];
  const int chunks = t.first[t.count];
  double s = 0.0;
  for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int q = tensor_of(t, c);
    const size_t at = (size_t)(c - t.first[q]) * t.chunk;
    const size_t n = min(t.n[q] - at, (size_t)t.chunk);
    s += t.bf16[q] ? square_sum(static_cast<const bf16_t*>(t.p[q]) + at, n)
                   : square_sum(static_cast<const float*>(t.p[q]) + at, n);
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

__global__ __launch_bounds__(kThreads) void grad_clip_kernel(GradTable t, const float* norm) {
  // (scale 1, or NaN: nothing to clip, so that values in place stay as they are)
  const float s = norm[1], scale = s < 1.0f ? s : 1.0f;
  const int chunks = t.first[t.count];
  for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int q = tensor_of(t, c);
    if (scale == 1.0f && t.p[q] == t.out[q]) continue;
    const size_t at = (size_t)(c - t.first[q]) * t.chunk;
    const size_t n = min(t.n[q] - at, (size_t)t.chunk);
    if (t.bf16[q])
      scale_to(static_cast<const bf16_t*>(t.p[q]) + at, static_cast<bf16_t*>(t.out[q]) + at, n, scale);
    else
      scale_to(static_cast<const float*>(t.p[q]) + at, static_cast<float*>(t.out[q]) + at, n, scale);
  }
}

// Values of a chunk, multiples of what 256 threads load at once.
int chunk_of(const moe_grad* g, int n) {
  size_t total = 0;
  for (int i = 0; i < n; ++i) total += g[i].n;
  return total < ((size_t)32 << 20) ? 4096 : 16384;
}

// Blocks of a launch of `chunks` chunks.
int chunk_blocks(int chunks) { return std::min(chunks, 8 * num_cus()); }

// f(table, blocks) for launches of up to kTensors tensors with values.
template <class F>
hipError_t for_tables(const moe_grad* g, int n, F&& f) {
  GradTable t;
  t.chunk = chunk_of(g, n);
  t.count = 0;
  t.first[0] = 0;
  for (int i = 0; i <= n; ++i) {
    const bool end = i == n;
    // (a launch's chunks are counted in 31 bits: a tensor that does not fit opens the next)
    const int64_t chunks = end ? 0 : (int64_t)((g[i].n + t.chunk - 1) / t.chunk);
    if (t.count > 0 && (end || t.count == kTensors || t.first[t.count] + chunks > INT32_MAX)) {
      if (const hipError_t e = f(t, chunk_blocks(t.first[t.count])); e != hipSuccess) return e;
      t.count = 0;
    }
    if (end || chunks == 0) continue;
    t.p[t.count] = g[i].grad;
    t.out[t.count] = g[i].out;
    t.n[t.count] = g[i].n;
    t.bf16[t.count] = g[i].dtype == MOE_BF16;
    t.first[t.count + 1] = t.first[t.count] + (int)chunks;
    ++t.count;
  }
  return hipSuccess;
}

}  // namespace

size_t grad_norm_ws_bytes(const moe_grad* g, int n) {
  size_t parts = 0;
  (void)for_tables(g, n, [&](const GradTable&, int blocks) {
    parts += blocks;
    return hipSuccess;
  });
  return parts * sizeof(double);
}

hipError_t launch_grad_norm(const moe_grad* g, int n, float max_norm, float* norm, void* ws,
                            hipStream_t s) {
  double* const part = static_cast<double*>(ws);
  int parts = 0;
  const hipError_t e = for_tables(g, n, [&](const GradTable& t, int blocks) {
    MOE_TIMED("grad_norm", s, grad_norm_kernel<<<blocks, kThreads, 0, s>>>(t, part + parts));
    parts += blocks;
    return hipGetLastError();
  });
  if (e != hipSuccess) return e;
  MOE_TIMED("grad_norm_sum", s, grad_norm_sum_kernel<<<1, 1024, 0, s>>>(part, parts, max_norm, norm));
  return hipGetLastError();
}

hipError_t launch_grad_clip(const moe_grad* g, int n, const float* norm, hipStream_t s) {
  return for_tables(g, n, [&](const GradTable& t, int blocks) {
    MOE_TIMED("grad_clip", s, grad_clip_kernel<<<blocks, kThreads, 0, s>>>(t, norm));
    return hipGetLastError();
  });
}

}  // namespace moe
