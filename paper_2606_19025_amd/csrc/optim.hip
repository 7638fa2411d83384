// Optimisers of the resident experts' fp32 master parameters.
//
// Sec. 3.4 ("Outer optimization"): every worker runs AdamW on its own
// parameters during the K local steps of a round and keeps the optimiser state
// across rounds, only for its own experts; at the round boundary the
// replica-group average of the pseudo-gradient is applied by a momentum outer
// optimiser (Alg. 2, OuterOpt).  App. F fixes the settings: AdamW with weight
// decay 0, betas (0.9, 0.95), eps 1e-8; DiLoCo's Nesterov outer step with
// learning rate 0.7 and momentum 0.9; LocalAdamW also averages the two moments
// over the replica group.
//
// All three are elementwise streams over fp32 arrays (HBM-bound): 16-byte
// vector accesses in a grid-stride loop over few blocks (stream_blocks), an
// element tail for n % 4.  Nothing
// is read twice, so the vector accesses are nontemporal (measured 14 % faster
// for AdamW than cached accesses).  Every
// operation is one IEEE fp32 rounding in a fixed order (no contraction into
// fused multiply-adds; division and square root correctly rounded), so the
// results are reproducible bit for bit by any fp32 evaluation of the same
// formulas.  The bf16 working copy that the grouped GEMMs read is written in
// the same pass (round to nearest even).
#include "common.h"
#include "kernels.h"
#include "timing.h"

#pragma clang fp contract(off)

namespace moe {
namespace {

struct AdamArgs {
  float* theta;
  const float* grad;
  float* m;
  float* v;
  bf16_t* theta_bf16;  // or NULL
  size_t n;
  float lr, b1, b2, eps, wd;
  float c1, c2;  // bias corrections 1 - beta^t of this step
};

// m' = b1 m + (1 - b1) g;  v' = b2 v + (1 - b2) g g;
// theta' = theta - lr ((m' / c1) / (sqrt(v' / c2) + eps) + wd theta)
// (contraction is off for this file; '/' and __builtin_sqrtf are the
// correctly rounded fp32 operations of HIP's default mode)
DEVI void adam_elem(const AdamArgs& a, float& th, float g, float& m, float& v) {
  const float om1 = 1.0f - a.b1, om2 = 1.0f - a.b2;
  m = a.b1 * m + om1 * g;
  v = a.b2 * v + om2 * (g * g);
  const float mh = m / a.c1;
  const float vh = v / a.c2;
  const float den = __builtin_sqrtf(vh) + a.eps;
  const float upd = mh / den + a.wd * th;
  th = th - a.lr * upd;
}

__global__ __launch_bounds__(256) void adamw_kernel(AdamArgs a) {
  const size_t n4 = a.n / 4;
  const size_t stride = (size_t)gridDim.x * 256;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n4; i += stride) {
    f32x4_t th = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(a.theta) + i);
    const f32x4_t g = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(a.grad) + i);
    f32x4_t m = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(a.m) + i);
    f32x4_t v = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(a.v) + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float t = th[e], mm = m[e], vv = v[e];
      adam_elem(a, t, g[e], mm, vv);
      th[e] = t; m[e] = mm; v[e] = vv;
    }
    __builtin_nontemporal_store(th, reinterpret_cast<f32x4_t*>(a.theta) + i);
    __builtin_nontemporal_store(m, reinterpret_cast<f32x4_t*>(a.m) + i);
    __builtin_nontemporal_store(v, reinterpret_cast<f32x4_t*>(a.v) + i);
    if (a.theta_bf16) {
      bf16x4_t o = {(bf16_t)th[0], (bf16_t)th[1], (bf16_t)th[2], (bf16_t)th[3]};
      reinterpret_cast<bf16x4_t*>(a.theta_bf16)[i] = o;
    }
  }
  for (size_t i = n4 * 4 + (size_t)blockIdx.x * 256 + threadIdx.x; i < a.n; i += stride) {
    float t = a.theta[i], mm = a.m[i], vv = a.v[i];
    adam_elem(a, t, a.grad[i], mm, vv);
    a.theta[i] = t; a.m[i] = mm; a.v[i] = vv;
    if (a.theta_bf16) a.theta_bf16[i] = (bf16_t)t;
  }
}

// AdamW over many tensors, gradients multiplied by the clip's scale first: a launch covers up to
// kAdamTensors tensors, whose table is a kernel argument; tensors are cut into chunks, which
// the blocks take in turn.  Bound by HBM, 28 bytes a value and 2 more for a bf16 copy: four tensors of 2^26
// values 1548 us (5.2 TB/s).  Many values: two blocks of large chunks a CU (seven streams a block; 156 M
// values 1114 us with one block, 1076 with two, 1128 with four); fewer: chunks of 1024 values to as many
// blocks as there are (200 tensors of 64 to 2^18 values 30 us less than in chunks of 8192; now 54).
constexpr int kAdamTensors = 72;
struct AdamTable {
  float* theta[kAdamTensors];
  const void* grad[kAdamTensors];
  float* m[kAdamTensors];
  float* v[kAdamTensors];
  bf16_t* low[kAdamTensors];  // or NULL
  float lr[kAdamTensors], wd[kAdamTensors];
  int first[kAdamTensors + 1];   // chunks before each tensor
  uint16_t tail[kAdamTensors];   // values of its last chunk, less one; top bit: a bf16 gradient
  int count, chunk;
  float b1, b2, eps, c1, c2;
};
static_assert(sizeof(AdamTable) <= 3968, "kernel arguments hold 4 KiB");

__global__ __launch_bounds__(256) void adamw_steps_kernel(AdamTable t, const float* norm) {
  const float scale = norm ? norm[1] : 1.0f;
  if (scale != scale) return;  // the gradients' norm is not finite: no step
  const int chunks = t.first[t.count];
  for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
    int q = 0;
    for (int hi = t.count - 1; q < hi;) {
      const int mid = (q + hi + 1) >> 1;
      if (t.first[mid] <= c) q = mid;
      else hi = mid - 1;
    }
    const size_t at = (size_t)(c - t.first[q]) * t.chunk;
    const unsigned tail = t.tail[q];
    const int n = c + 1 < t.first[q + 1] ? t.chunk : (int)(tail & 0x7fff) + 1, n4 = n / 4;
    float* const th = t.theta[q] + at;
    float* const m = t.m[q] + at;
    float* const v = t.v[q] + at;
    bf16_t* const low = t.low[q] ? t.low[q] + at : nullptr;
    const bool bf16 = tail >> 15;
    const float* const g = static_cast<const float*>(t.grad[q]) + (bf16 ? 0 : at);
    const bf16_t* const gb = static_cast<const bf16_t*>(t.grad[q]) + (bf16 ? at : 0);
    AdamArgs a{};
    a.lr = t.lr[q]; a.wd = t.wd[q];
    a.b1 = t.b1; a.b2 = t.b2; a.eps = t.eps; a.c1 = t.c1; a.c2 = t.c2;
    for (int i = threadIdx.x; i < n4; i += 256) {
      f32x4_t tt = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(th) + i);
      f32x4_t mm = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(m) + i);
      f32x4_t vv = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(v) + i);
      f32x4_t gg;
      if (bf16) gg = __builtin_convertvector(reinterpret_cast<const bf16x4_t*>(gb)[i], f32x4_t);
      else gg = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(g) + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float x = tt[e], y = mm[e], z = vv[e];
        adam_elem(a, x, gg[e] * scale, y, z);
        tt[e] = x; mm[e] = y; vv[e] = z;
      }
      __builtin_nontemporal_store(tt, reinterpret_cast<f32x4_t*>(th) + i);
      __builtin_nontemporal_store(mm, reinterpret_cast<f32x4_t*>(m) + i);
      __builtin_nontemporal_store(vv, reinterpret_cast<f32x4_t*>(v) + i);
      if (low) reinterpret_cast<bf16x4_t*>(low)[i] = __builtin_convertvector(tt, bf16x4_t);
    }
    for (int i = n4 * 4 + threadIdx.x; i < n; i += 256) {
      float x = th[i], y = m[i], z = v[i];
      adam_elem(a, x, (bf16 ? (float)gb[i] : g[i]) * scale, y, z);
      th[i] = x; m[i] = y; v[i] = z;
      if (low) low[i] = (bf16_t)x;
    }
  }
}

struct OuterArgs {
  float* start;
  float* now;
  const float* delta;
  float* mom;
  bf16_t* theta_bf16;  // or NULL
  size_t n;
  float lr, mu;
};

// b' = mu b + delta;  theta' = start - lr (delta + mu b'); start = now = theta'
DEVI float outer_elem(const OuterArgs& a, float start, float delta, float& b) {
  b = a.mu * b + delta;
  const float upd = delta + a.mu * b;
  return start - a.lr * upd;
}

__global__ __launch_bounds__(256) void outer_nesterov_kernel(OuterArgs a) {
  const size_t n4 = a.n / 4;
  const size_t stride = (size_t)gridDim.x * 256;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n4; i += stride) {
    const f32x4_t s = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(a.start) + i);
    const f32x4_t d = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(a.delta) + i);
    f32x4_t b = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(a.mom) + i);
    f32x4_t th;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float bb = b[e];
      th[e] = outer_elem(a, s[e], d[e], bb);
      b[e] = bb;
    }
    __builtin_nontemporal_store(b, reinterpret_cast<f32x4_t*>(a.mom) + i);
    __builtin_nontemporal_store(th, reinterpret_cast<f32x4_t*>(a.start) + i);
    __builtin_nontemporal_store(th, reinterpret_cast<f32x4_t*>(a.now) + i);
    if (a.theta_bf16) {
      bf16x4_t o = {(bf16_t)th[0], (bf16_t)th[1], (bf16_t)th[2], (bf16_t)th[3]};
      reinterpret_cast<bf16x4_t*>(a.theta_bf16)[i] = o;
    }
  }
  for (size_t i = n4 * 4 + (size_t)blockIdx.x * 256 + threadIdx.x; i < a.n; i += stride) {
    float bb = a.mom[i];
    const float th = outer_elem(a, a.start[i], a.delta[i], bb);
    a.mom[i] = bb;
    a.start[i] = th;
    a.now[i] = th;
    if (a.theta_bf16) a.theta_bf16[i] = (bf16_t)th;
  }
}

struct MeanArgs {
  const float* local;
  const float* peers[kMaxPeers];
  float* out;
  size_t n;
  int n_peers;
  float scale;
};

// out = (((local + p_0) + p_1) + ...) * fp32(1 / (n_peers + 1))
__global__ __launch_bounds__(256) void replica_mean_kernel(MeanArgs a) {
  const size_t n4 = a.n / 4;
  const size_t stride = (size_t)gridDim.x * 256;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n4; i += stride) {
    f32x4_t acc = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(a.local) + i);
    for (int p = 0; p < a.n_peers; ++p)
      acc = acc + __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(a.peers[p]) + i);
    __builtin_nontemporal_store(acc * a.scale, reinterpret_cast<f32x4_t*>(a.out) + i);
  }
  for (size_t i = n4 * 4 + (size_t)blockIdx.x * 256 + threadIdx.x; i < a.n; i += stride) {
    float acc = a.local[i];
    for (int p = 0; p < a.n_peers; ++p) acc = acc + a.peers[p][i];
    a.out[i] = acc * a.scale;
  }
}

}  // namespace

hipError_t launch_adamw(float* theta, const float* grad, float* m, float* v, size_t n, float lr,
                        float beta1, float beta2, float eps, float wd, float c1, float c2,
                        void* theta_bf16, hipStream_t s) {
  if (n == 0) return hipSuccess;
  AdamArgs a{theta, grad, m, v, static_cast<bf16_t*>(theta_bf16), n, lr, beta1, beta2, eps, wd,
             c1, c2};
  MOE_TIMED("adamw_step", s, adamw_kernel<<<stream_blocks(n, kFewBlocks, n >= (64u << 20) ? 1 : 2), 256, 0, s>>>(a));
  return hipGetLastError();
}

hipError_t launch_adamw_steps(const moe_adamw_tensor* p, int n, float lr, float beta1, float beta2,
                              float eps, float c1, float c2, const float* norm, hipStream_t s) {
  AdamTable t;
  t.b1 = beta1; t.b2 = beta2; t.eps = eps; t.c1 = c1; t.c2 = c2;
  size_t total = 0;
  for (int i = 0; i < n; ++i) total += p[i].n;
  const bool few = total >= kFewBlocks;
  t.chunk = few ? 8192 : 1024;
  t.count = 0;
  t.first[0] = 0;
  for (int i = 0; i <= n; ++i) {
    const bool end = i == n;
    // (a launch's chunks, and a block's steps past the last of them, are counted in 31 bits: a tensor that
    // does not fit opens the next)
    const int64_t chunks = end ? 0 : (int64_t)((p[i].n + t.chunk - 1) / t.chunk);
    if (t.count > 0 && (end || t.count == kAdamTensors || t.first[t.count] + chunks > 1 << 30)) {
      const int blocks = std::min(t.first[t.count], few ? 2 * num_cus() : 8192);
      MOE_TIMED("adamw_steps", s, adamw_steps_kernel<<<blocks, 256, 0, s>>>(t, norm));
      if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
      t.count = 0;
    }
    if (end || chunks == 0) continue;
    const int k = t.count++;
    t.theta[k] = p[i].theta; t.grad[k] = p[i].grad; t.m[k] = p[i].m; t.v[k] = p[i].v;
    t.low[k] = static_cast<bf16_t*>(p[i].theta_bf16);
    t.lr[k] = lr * p[i].lr_scale;
    t.wd[k] = p[i].weight_decay;
    t.tail[k] = (uint16_t)((p[i].n - 1) % t.chunk | (p[i].grad_dtype == MOE_BF16 ? 0x8000 : 0));
    t.first[k + 1] = t.first[k] + (int)chunks;
  }
  return hipSuccess;
}

hipError_t launch_outer_nesterov(float* start, float* now, const float* delta, float* mom,
                                 size_t n, float lr, float mu, void* theta_bf16, hipStream_t s) {
  if (n == 0) return hipSuccess;
  OuterArgs a{start, now, delta, mom, static_cast<bf16_t*>(theta_bf16), n, lr, mu};
  MOE_TIMED("outer_nesterov", s, outer_nesterov_kernel<<<stream_blocks(n, kFewBlocks, 1), 256, 0, s>>>(a));
  return hipGetLastError();
}

hipError_t launch_replica_mean(const float* local, const float* const* peers, int n_peers,
                               size_t n, float* out, hipStream_t s) {
  if (n == 0) return hipSuccess;
  MeanArgs a{};
  a.local = local;
  for (int p = 0; p < n_peers; ++p) a.peers[p] = peers[p];
  a.out = out;
  a.n = n;
  a.n_peers = n_peers;
  a.scale = 1.0f / (float)(n_peers + 1);
  MOE_TIMED("replica_mean", s, replica_mean_kernel<<<peer_stream_blocks(n, n_peers, 5), 256, 0, s>>>(a));
  return hipGetLastError();
}

}  // namespace moe
