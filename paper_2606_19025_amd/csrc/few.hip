// The few-token layer (few.h): the logits, and the host's side.
#include "few.h"

namespace moe {
namespace {

constexpr int LW = 8;  // waves of few_logits_bf16_kernel: the router's shares of d

// bf16: LT tokens by LE experts per block.  The sums are the router's, to the bit: wave w
// takes the 64-wide slices w, w + 8, ... of d on v_mfma_f32_32x32x16_bf16 with the same
// sixteen k in each, and the waves' sums are added in order.  Most of the instruction's rows
// are empty: a block's time is that of its loads, and with 8 by 8 many CUs share them
// (48 tokens, d = 2048, 64 experts: with 32 tokens 5 us, so 2).
constexpr int LE = 8, LT = 8;
__global__ __launch_bounds__(64 * LW) void few_logits_bf16_kernel(FewArgs a) {
  __shared__ float part[LW][LT * LE];
  const bf16_t* x = static_cast<const bf16_t*>(a.x);
  const bf16_t* w = static_cast<const bf16_t*>(a.w_router);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = lane & 31, half = lane >> 5;
  const int e0 = blockIdx.x * LE, t0 = blockIdx.y * LT;
  const int n = (a.d + 63) / 64;
  const bool has_t = row < LT && t0 + row < a.T, has_e = row < LE && e0 + row < a.E;
  const bf16_t* xr = x + (size_t)(has_t ? t0 + row : 0) * a.d;
  const bf16_t* wr = w + (size_t)(has_e ? e0 + row : 0) * a.d;
  f32x16_t acc = {};
  const bf16x8_t zero = {};
  constexpr int U = 4;
  for (int s0 = wave; s0 < n; s0 += U * LW) {
    bf16x8_t xv[U][4], wv[U][4];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = (s0 + u * LW) * 64 + half * 32 + q * 8;
        xv[u][q] = has_t && c < a.d ? *reinterpret_cast<const bf16x8_t*>(xr + c) : zero;
        wv[u][q] = has_e && c < a.d ? *reinterpret_cast<const bf16x8_t*>(wr + c) : zero;
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xv[u][q], wv[u][q], acc, 0, 0, 0);
  }
  if (row < LE)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int i = (r >> 2) * 8 + half * 4 + (r & 3);
      if (i < LT) part[wave][i * LE + row] = acc[r];
    }
  __syncthreads();
  if (threadIdx.x < LT * LE) {
    const int t = t0 + threadIdx.x / LE, e = e0 + threadIdx.x % LE;
    float v = part[0][threadIdx.x];
#pragma unroll
    for (int q = 1; q < LW; ++q) v += part[q][threadIdx.x];
    if (t < a.T && e < a.E) {
      if (a.bias) v += a.bias[e];
      a.logits[(size_t)t * a.E + e] = v * a.inv_tau;
    }
  }
}

// fp32: 16 tokens by 16 experts per block, a logit per thread as one chain of fused
// multiply-adds in the order of d (the router's bits).  Chunks of 64 of d go through LDS,
// the next one on its way meanwhile.
__global__ __launch_bounds__(256) void few_logits_f32_kernel(FewArgs a) {
  constexpr int C = 64, S = C + 4;
  __shared__ float xs[16][S], ws[16][S];
  const float* x = static_cast<const float*>(a.x);
  const float* w = static_cast<const float*>(a.w_router);
  const int e0 = blockIdx.x * 16, t0 = blockIdx.y * 16;
  const int lr = threadIdx.x >> 4, lc = (threadIdx.x & 15) * 4;  // the thread's 16 bytes of a chunk
  const float* xp = x + (size_t)min(t0 + lr, a.T - 1) * a.d;
  const float* wp = w + (size_t)min(e0 + lr, a.E - 1) * a.d;
  const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
  auto at = [&](const float* p, int c) { return c < a.d ? *reinterpret_cast<const f32x4_t*>(p + c) : zero; };
  f32x4_t xv = at(xp, lc), wv = at(wp, lc);
  const int i = threadIdx.x >> 4, j = threadIdx.x & 15;
  float v = 0.f;
  for (int c = 0; c < a.d; c += C) {
    *reinterpret_cast<f32x4_t*>(&xs[lr][lc]) = xv;
    *reinterpret_cast<f32x4_t*>(&ws[lr][lc]) = wv;
    __syncthreads();
    xv = at(xp, c + C + lc);
    wv = at(wp, c + C + lc);
#pragma unroll
    for (int q = 0; q < C; q += 4) {
      const f32x4_t p = *reinterpret_cast<const f32x4_t*>(&xs[i][q]);
      const f32x4_t r = *reinterpret_cast<const f32x4_t*>(&ws[j][q]);
#pragma unroll
      for (int s = 0; s < 4; ++s) v = fmaf(p[s], r[s], v);
    }
    __syncthreads();
  }
  const int t = t0 + i, e = e0 + j;
  if (t < a.T && e < a.E) {
    if (a.bias) v += a.bias[e];
    a.logits[(size_t)t * a.E + e] = v * a.inv_tau;
  }
}

size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

struct FewLayout {
  size_t local, logits, h, hs, bytes;
};
FewLayout few_layout(const moe_few* f) {
  FewLayout l;
  const size_t e = f->dtype == MOE_BF16 ? 2 : 4, T = f->T;
  size_t at = 0;
  auto take = [&](size_t n) { const size_t o = at; at += up256(n); return o; };
  l.local = take(T * f->k * 4);
  l.logits = take(f->logits ? 0 : T * f->E * 4);
  l.h = take(T * f->k * f->H * e);
  l.hs = take(T * f->Hs * e);
  l.bytes = at;
  return l;
}

}  // namespace

size_t few_ws_bytes(const moe_few* f) { return few_layout(f).bytes; }

hipError_t launch_few(const moe_few* f, hipStream_t s) {
  if (f->T == 0) return hipSuccess;
  const FewLayout l = few_layout(f);
  char* ws = static_cast<char*>(f->ws);
  FewArgs a{};
  a.x = f->x; a.w_router = f->w_router; a.bias = f->router_bias; a.resident = f->resident;
  a.wgu = f->w_gate_up; a.wd = f->w_down; a.sgu = f->shared_gate_up; a.sd = f->shared_down;
  a.wgu_s = f->w_gate_up_scales; a.wd_s = f->w_down_scales;
  a.sgu_s = f->shared_gate_up_scales; a.sd_s = f->shared_down_scales;
  a.logits = f->logits ? f->logits : reinterpret_cast<float*>(ws + l.logits);
  a.idx = f->topk_idx; a.tw = f->topk_w; a.local = f->topk_local; a.y = f->y;
  a.w_local = reinterpret_cast<int32_t*>(ws + l.local);
  a.h = ws + l.h;
  a.hs = ws + l.hs;
  a.T = f->T; a.d = f->d; a.E = f->E; a.k = f->k; a.E_r = f->E_r; a.H = f->H; a.Hs = f->Hs;
  a.gate = f->gate; a.inv_tau = f->inv_tau;
  if (f->dtype == MOE_BF16)
    MOE_TIMED("few_logits", s, few_logits_bf16_kernel<<<dim3(ceil_div(f->E, LE), ceil_div(f->T, LT)),
                                                        64 * LW, 0, s>>>(a));
  else
    MOE_TIMED("few_logits", s, few_logits_f32_kernel<<<dim3(ceil_div(f->E, 16), ceil_div(f->T, 16)),
                                                       256, 0, s>>>(a));
  const bool swiglu = f->activation == MOE_ACT_SWIGLU;
  if (f->weights == MOE_W_MXFP4) run_few_mx(a, swiglu, s);
  else if (f->dtype == MOE_BF16) run_few_bf16(a, swiglu, s);
  else run_few_f32(a, swiglu, s);
  return hipGetLastError();
}

}  // namespace moe
