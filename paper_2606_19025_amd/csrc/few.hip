// The whole MoE layer for a few tokens (T <= 64): evaluation and generation.
//
//   z = (x Wr^T + b) / tau, top-k, gates           (as the router, to the bit)
//   h_tj = s_tj act(Wgu_e x_t)                      for each resident route (t, j) to expert e
//   y_t  = sum_j Wd_e h_tj + Wd_s act(Wgu_s x_t)    (s: the shared experts, gate 1)
//
// Bound by HBM: every active expert's weights are read once, for a handful of tokens each.
// Three launches: the logits (few_logits_*), the first projections (few_gu_kernel) and the
// second ones with the sum over experts (few_down_kernel).  No rows are moved: the weights
// are the matrix instruction's first operand (16 rows of an expert's matrix) and the tokens
// its second (16 columns, all of the batch's tokens in up to four tiles; a tile that no
// token of an expert falls in is skipped).  Columns of tokens that are not routed to the
// expert cost nothing that counts: in few_gu_kernel they are not stored, in
// few_down_kernel they are zeros.  So the second kernel's accumulators run on from expert
// to expert, with the gate already in h.
//
// Weights go from HBM to registers in the order of the instruction's operand: a lane
// takes a row's consecutive bytes, the four lanes of a row 64 or 128 of them.  (The
// order of k within an instruction is free as long as both operands have the same.)
#include <type_traits>

#include "kernels.h"
#include "mx.h"
#include "route_select.h"
#include "timing.h"

namespace moe {
namespace {

constexpr int LW = 8;              // waves of few_logits_bf16_kernel: the router's shares of d
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
  void* h;         // [T k, H], rows of resident routes
  void* hs;        // [T, Hs]
  int T, d, E, k, E_r, H, Hs, gate;
  float inv_tau;
};

// ------------------------------------------------------------------ logits
// bf16: 32 tokens by LE experts per block.  The sums are the router's, to the bit: wave w
// takes the 64-wide slices w, w + 8, ... of d on v_mfma_f32_32x32x16_bf16 with the same
// sixteen k in each, and the waves' sums are added in order.  Few experts per block, so
// that a single token's logits come from many CUs.
constexpr int LE = 8;
__global__ __launch_bounds__(64 * LW) void few_logits_bf16_kernel(FewArgs a) {
  __shared__ float part[LW][32 * LE];
  const bf16_t* x = static_cast<const bf16_t*>(a.x);
  const bf16_t* w = static_cast<const bf16_t*>(a.w_router);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = lane & 31, half = lane >> 5;
  const int e0 = blockIdx.x * LE, t0 = blockIdx.y * 32;
  const int n = (a.d + 63) / 64;
  const bool has_t = t0 + row < a.T, has_e = row < LE && e0 + row < a.E;
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
      part[wave][i * LE + row] = acc[r];
    }
  __syncthreads();
  if (threadIdx.x < 32 * LE) {
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

// ------------------------------------------------------------------ routes
// The block's tables: each route's gate and local expert, the experts that any token is
// routed to (in order), and for each of those the route of every token (or -1).
struct FewTables {
  float gate[FEW_T * FEW_K];
  int16_t local[FEW_T * FEW_K];
  int16_t expert[256];        // active expert -> local id
  int16_t slot[256];          // local id -> active expert, or -1
  int lmap[256];
  int n_active;
};

// Top-k, gates and local ids of token t, by 16 lanes (the router's selection on logits in
// global memory): lane s of a group holds the experts s, s + 16, ...
template <int NE>
DEVI void few_select(const FewArgs& a, FewTables& tb, int t, bool publish) {
  const int lane = threadIdx.x & 63, s = lane & 15;
  const float* z = a.logits + (size_t)t * a.E;
  const bool has = t < a.T;
  float v[NE];
  uint64_t cand[NE];
#pragma unroll
  for (int q = 0; q < NE; ++q) {
    const int e = q * 16 + s;
    v[q] = has && e < a.E ? sel_value(z[e]) : 0.f;
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
    // (a resident set larger than E_r says: its last experts are ghosts here)
    const int l = tb.lmap[my_id] < a.E_r ? tb.lmap[my_id] : -1;
    tb.gate[o] = g;
    tb.local[o] = (int16_t)l;
    if (publish) {
      a.w_local[o] = l;
      if (a.idx) a.idx[o] = my_id;
      if (a.tw) a.tw[o] = g;
      if (a.local) a.local[o] = l;
    }
  }
}

// The active experts in ascending order (one wave; slot[] holds 1 for an expert with a route).
DEVI void few_active(const FewArgs& a, FewTables& tb) {
  const int lane = threadIdx.x & 63;
  int n = 0;
  for (int r0 = 0; r0 < a.E_r; r0 += 64) {
    const int r = r0 + lane;
    const bool on = r < a.E_r && tb.slot[r] != 0;
    const uint64_t m = __ballot(on);
    const int s = n + __popcll(m & ((1ull << lane) - 1ull));
    if (r < a.E_r) tb.slot[r] = (int16_t)(on ? s : -1);
    if (on) tb.expert[s] = (int16_t)r;
    n += __popcll(m);
  }
  if (lane == 0) tb.n_active = n;
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
// One step of a wave: 16 weight rows by KS of k.  Lane (r, q) = (lane % 16, lane / 16)
// holds the KL = KS / 4 values of row r from k0 + q KL on, and of token r likewise.
//   bf16   KL 16 (32 bytes), two v_mfma_f32_16x16x32_bf16
//   fp32   KL 8 (32 bytes), eight v_mfma_f32_16x16x4_f32
//   MXFP4  KL 32 (16 bytes and one scale), widened to bf16 (exactly, a value has two
//          significant bits): four v_mfma_f32_16x16x32_bf16 on bf16 activations
template <class E, bool MX> struct Op;
template <> struct Op<bf16_t, false> {
  static constexpr int KL = 16;
  struct W { bf16x8_t v[2]; };
  struct X { bf16x8_t v[2]; };
  DEVI static void load(W& w, const void* p, const uint8_t*, size_t row, int K, int k, bool ok) {
    const bf16_t* q = static_cast<const bf16_t*>(p) + row * K + k;
    const bf16x8_t z = {};
    w.v[0] = ok ? *reinterpret_cast<const bf16x8_t*>(q) : z;
    w.v[1] = ok ? *reinterpret_cast<const bf16x8_t*>(q + 8) : z;
  }
  DEVI static void load_x(X& x, const bf16_t* q, bool ok) {
    const bf16x8_t z = {};
    x.v[0] = ok ? *reinterpret_cast<const bf16x8_t*>(q) : z;
    x.v[1] = ok ? *reinterpret_cast<const bf16x8_t*>(q + 8) : z;
  }
  DEVI static f32x4_t mma(const W& w, const X& x, f32x4_t c) {
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.v[0], x.v[0], c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.v[1], x.v[1], c, 0, 0, 0);
  }
};
template <> struct Op<float, false> {
  static constexpr int KL = 8;
  struct W { f32x4_t v[2]; };
  struct X { f32x4_t v[2]; };
  DEVI static void load(W& w, const void* p, const uint8_t*, size_t row, int K, int k, bool ok) {
    load_x(w, static_cast<const float*>(p) + row * K + k, ok);
  }
  template <class V> DEVI static void load_x(V& x, const float* q, bool ok) {
    const f32x4_t z = {0.f, 0.f, 0.f, 0.f};
    x.v[0] = ok ? *reinterpret_cast<const f32x4_t*>(q) : z;
    x.v[1] = ok ? *reinterpret_cast<const f32x4_t*>(q + 4) : z;
  }
  DEVI static f32x4_t mma(const W& w, const X& x, f32x4_t c) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(w.v[i >> 2][i & 3], x.v[i >> 2][i & 3], c, 0, 0, 0);
    return c;
  }
};
typedef __bf16 bf16x2_v __attribute__((ext_vector_type(2)));
template <> struct Op<bf16_t, true> {
  static constexpr int KL = 32;
  struct W { u32x4_t c; unsigned s; };
  struct X { bf16x8_t v[4]; };
  DEVI static void load(W& w, const void* p, const uint8_t* s, size_t row, int K, int k, bool ok) {
    const u32x4_t z = {0u, 0u, 0u, 0u};
    w.c = ok ? *reinterpret_cast<const u32x4_t*>(static_cast<const uint8_t*>(p) + (row * K + k) / 2) : z;
    w.s = ok ? s[row * mx_stride(K) + k / MX_BLOCK] : 0u;
  }
  DEVI static void load_x(X& x, const bf16_t* q, bool ok) {
    const bf16x8_t z = {};
#pragma unroll
    for (int i = 0; i < 4; ++i) x.v[i] = ok ? *reinterpret_cast<const bf16x8_t*>(q + 8 * i) : z;
  }
  DEVI static bf16x8_t widen(unsigned c, float s) {
    const bf16x2_v a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0);
    const bf16x2_v b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1);
    const bf16x2_v d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2);
    const bf16x2_v e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3);
    const bf16x8_t v = {a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
    return v;
  }
  DEVI static f32x4_t mma(const W& w, const X& x, f32x4_t c) {
    const float s = mx_scale_f32(w.s);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(w.c[i], s), x.v[i], c, 0, 0, 0);
    return c;
  }
};

// ------------------------------------------------------------------ first projections
// An item is 16 hidden units of one expert (32 rows of a SwiGLU expert's matrix, 16 of a
// SiLU one's); its k is dealt over the block's waves in steps, and the waves' sums are
// added in order through LDS.
//
// The shared experts' items come first and need no routing; every block makes the routes'
// tables itself when it comes to its first routed item (a launch of its own for them would
// take longer than their two microseconds).
constexpr int gu_waves(int NT) { return NT == 1 ? 4 : 8; }

template <class E, bool MX, int ACT, int NT>
__global__ __launch_bounds__(64 * gu_waves(NT), NT == 1 ? 4 : 2) void few_gu_kernel(FewArgs a) {
  using O = Op<E, MX>;
  constexpr int FW = gu_waves(NT), FT = 64 * FW;
  constexpr int KL = O::KL, KS = 4 * KL;
  constexpr int R = ACT == MOE_ACT_SWIGLU ? 2 : 1;
  constexpr int U = NT == 1 && !MX ? 4 : 2;  // steps whose loads are issued together
  __shared__ FewTables tb;
  __shared__ f32x4_t red[FW][R][NT][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int l16 = lane & 15, q4 = lane >> 4;
  const E* x = static_cast<const E*>(a.x);

  // hidden units h0 .. h0 + 15 of one expert; my_p: the row of h for lane t's token, or -1
  auto item = [&](bool shared, int r, int h0, int my_p) {
    const int H = shared ? a.Hs : a.H;
    const uint64_t who = __ballot(my_p >= 0);
    const void* W = shared ? a.sgu : a.wgu;
    const uint8_t* S = shared ? a.sgu_s : a.wgu_s;
    const size_t row0 = (size_t)r * R * H + h0 + l16;
    f32x4_t acc[R][NT];
#pragma unroll
    for (int g = 0; g < R; ++g)
#pragma unroll
      for (int n = 0; n < NT; ++n) acc[g][n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int k0 = wave * KS; k0 < a.d; k0 += U * FW * KS) {
      typename O::W w[U][R];
      typename O::X xv[U][NT];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int k = k0 + u * FW * KS + q4 * KL;
        const bool ok = k < a.d;
#pragma unroll
        for (int g = 0; g < R; ++g) O::load(w[u][g], W, S, row0 + (size_t)g * H, a.d, k, ok);
#pragma unroll
        for (int n = 0; n < NT; ++n)
          O::load_x(xv[u][n], x + (size_t)(16 * n + l16) * a.d + k, ok && (who >> (16 * n + l16) & 1));
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int g = 0; g < R; ++g)
#pragma unroll
          for (int n = 0; n < NT; ++n) acc[g][n] = O::mma(w[u][g], xv[u][n], acc[g][n]);
    }
    __syncthreads();  // the previous item's sums have been read
#pragma unroll
    for (int g = 0; g < R; ++g)
#pragma unroll
      for (int n = 0; n < NT; ++n) red[wave][g][n][lane] = acc[g][n];
    __syncthreads();
    if (wave < NT) {
      // this wave's tile: token 16 wave + l16, hidden units h0 + 4 q4 ..
      const int t = 16 * wave + l16;
      f32x4_t v[R];
#pragma unroll
      for (int g = 0; g < R; ++g) {
        v[g] = red[0][g][wave][lane];
#pragma unroll
        for (int q = 1; q < FW; ++q) v[g] += red[q][g][wave][lane];
      }
      const int p = __shfl(my_p, t & 63, 64);
      if (t < a.T && p >= 0) {
        const float gate = shared ? 1.0f : tb.gate[p];
        E* out = static_cast<E*>(shared ? a.hs : a.h) + (size_t)p * H + h0 + 4 * q4;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float s = gate * silu_f(v[0][i]);
          out[i] = from_f32<E>(R == 2 ? s * v[R - 1][i] : s);
        }
      }
    }
  };

  const int n_s = a.Hs / 16, n_r = a.H / 16;
  int it = blockIdx.x;
  for (; it < n_s; it += gridDim.x) item(true, 0, it * 16, lane < a.T ? lane : -1);

  if (wave == 0) build_local_map(a.resident, a.E, tb.lmap);
  for (int i = threadIdx.x; i < 256; i += FT) tb.slot[i] = 0;
  __syncthreads();
  for (int t = wave * 4 + q4; t - q4 < a.T; t += FW * 4) {
    if (a.E <= 64) few_select<4>(a, tb, t, blockIdx.x == 0);
    else if (a.E <= 128) few_select<8>(a, tb, t, blockIdx.x == 0);
    else few_select<16>(a, tb, t, blockIdx.x == 0);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.T * a.k; i += FT)
    if (tb.local[i] >= 0) tb.slot[tb.local[i]] = 1;
  __syncthreads();
  if (wave == 0) few_active(a, tb);
  __syncthreads();
  for (; it < n_s + tb.n_active * n_r; it += gridDim.x) {
    const int r = tb.expert[(it - n_s) / n_r];
    item(false, r, (it - n_s) % n_r * 16, route_to(a, tb, lane, r));
  }
}

// ------------------------------------------------------------------ second projections
// A block is RB columns of y (rows of W_d; the matrix instruction's other rows are empty)
// and the whole reduction: the shared experts' hidden units, then all active experts', in
// steps of which each wave takes consecutive ones.  Sums run on over experts; the waves'
// are added in order through LDS.  RB is 16, or less where that would leave CUs without a
// block: cutting the reduction into parts instead, added by the last block to finish, took
// three times as long (the fences write back each XCD's whole L2).
constexpr int DW = 16;  // waves

template <class E, bool MX, int NT, int RB>
__global__ __launch_bounds__(64 * DW) void few_down_kernel(FewArgs a) {
  using O = Op<E, MX>;
  constexpr int KL = O::KL, KS = 4 * KL;
  constexpr int U = NT == 1 && !MX ? 2 : 1;  // steps in a stage; two stages' loads in flight
  __shared__ FewTables tb;
  __shared__ f32x4_t red[DW][NT][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int l16 = lane & 15, q4 = lane >> 4;
  for (int i = threadIdx.x; i < a.T * a.k; i += 64 * DW) tb.local[i] = (int16_t)a.w_local[i];
  for (int i = threadIdx.x; i < 256; i += 64 * DW) tb.slot[i] = 0;
  const int row = blockIdx.x * RB + l16;
  const bool has_row = l16 < RB;
  f32x4_t acc[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) acc[n] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  struct Stage {
    typename O::W w[U];
    typename O::X x[U][NT];
  };
  int cur = -1, my_p = -1, r = 0;  // the active expert at hand and lane t's route to it
  // the steps [s0, s1) of n_h to an expert; the shared ones if SH
  auto run = [&](auto SH, int s0, int s1, int n_h) {
    constexpr bool shared = decltype(SH)::value;
    const int H = shared ? a.Hs : a.H;
    const void* W = shared ? a.sd : a.wd;
    const uint8_t* S = shared ? a.sd_s : a.wd_s;
    const E* h = static_cast<const E*>(shared ? a.hs : a.h);
    auto load = [&](Stage& g, int s) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int st = s + u;
        const bool on = st < s1;
        int k = st;
        if constexpr (!shared) {
          const int act = st / n_h;
          k -= act * n_h;
          if (on && act != cur) {
            cur = act;
            r = tb.expert[act];
            my_p = route_to(a, tb, lane, r);
          }
        }
        k = k * KS + q4 * KL;
        const bool ok = on && k < H;
        O::load(g.w[u], W, S, (size_t)r * a.d + row, H, k, ok && has_row);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const int p = __shfl(my_p, 16 * n + l16, 64);
          O::load_x(g.x[u][n], h + (size_t)(p < 0 ? 0 : p) * H + k, ok && p >= 0);
        }
      }
    };
    auto mma = [&](const Stage& g) {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[n] = O::mma(g.w[u], g.x[u][n], acc[n]);
    };
    if (s0 >= s1) return;
    Stage g0, g1;
    load(g0, s0);
    for (int s = s0; s < s1; s += 2 * U) {
      load(g1, s + U);
      mma(g0);
      load(g0, s + 2 * U);
      mma(g1);
    }
  };
  if (a.Hs) {
    my_p = lane < a.T ? lane : -1;
    const int n = ceil_div(a.Hs, KS);
    run(std::true_type{}, n * wave / DW, n * (wave + 1) / DW, n);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.T * a.k; i += 64 * DW)
    if (tb.local[i] >= 0) tb.slot[tb.local[i]] = 1;
  __syncthreads();
  if (wave == 0) few_active(a, tb);
  __syncthreads();
  const int n_h = ceil_div(a.H, KS), n = tb.n_active * n_h;
  run(std::false_type{}, n * wave / DW, n * (wave + 1) / DW, n_h);
#pragma unroll
  for (int q = 0; q < NT; ++q) red[wave][q][lane] = acc[q];
  __syncthreads();
  // token t of tile `wave`, columns RB blockIdx.x + 4 q4 ..
  const int t = 16 * wave + l16;
  if (wave < NT && t < a.T && 4 * q4 < RB) {
    f32x4_t v = red[0][wave][lane];
#pragma unroll
    for (int q = 1; q < DW; ++q) v += red[q][wave][lane];
    E* y = static_cast<E*>(a.y) + (size_t)t * a.d + blockIdx.x * RB + 4 * q4;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = from_f32<E>(v[i]);
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

template <class E, bool MX, int ACT, int NT>
void few_launch(const FewArgs& a, hipStream_t s) {
  const int64_t items = std::min<int64_t>(a.E_r, (int64_t)a.T * a.k) * (a.H / 16) + a.Hs / 16;
  const int most = (NT == 1 ? 4 : 2) * num_cus();  // as many as are resident at once
  MOE_TIMED("few_gu", s, few_gu_kernel<E, MX, ACT, NT>
            <<<(int)std::max<int64_t>(1, std::min<int64_t>(items, most)), 64 * gu_waves(NT), 0, s>>>(a));
#define FEW_DOWN(RB) \
  MOE_TIMED("few_down", s, few_down_kernel<E, MX, NT, RB><<<a.d / RB, 64 * DW, 0, s>>>(a))
  if (a.d / 16 >= num_cus()) FEW_DOWN(16);
  else if (a.d / 8 >= num_cus()) FEW_DOWN(8);
  else FEW_DOWN(4);
#undef FEW_DOWN
}
template <class E, bool MX, int ACT>
void few_tiles(const FewArgs& a, hipStream_t s) {
  if (a.T <= 16) few_launch<E, MX, ACT, 1>(a, s);
  else if (a.T <= 32) few_launch<E, MX, ACT, 2>(a, s);
  else if (a.T <= 48) few_launch<E, MX, ACT, 3>(a, s);
  else few_launch<E, MX, ACT, 4>(a, s);
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
    MOE_TIMED("few_logits", s, few_logits_bf16_kernel<<<dim3(ceil_div(f->E, LE), ceil_div(f->T, 32)),
                                                        64 * LW, 0, s>>>(a));
  else
    MOE_TIMED("few_logits", s, few_logits_f32_kernel<<<dim3(ceil_div(f->E, 16), ceil_div(f->T, 16)),
                                                       256, 0, s>>>(a));
  const bool swiglu = f->activation == MOE_ACT_SWIGLU;
  if (f->weights == MOE_W_MXFP4)
    swiglu ? few_tiles<bf16_t, true, MOE_ACT_SWIGLU>(a, s) : few_tiles<bf16_t, true, MOE_ACT_SILU>(a, s);
  else if (f->dtype == MOE_BF16)
    swiglu ? few_tiles<bf16_t, false, MOE_ACT_SWIGLU>(a, s) : few_tiles<bf16_t, false, MOE_ACT_SILU>(a, s);
  else
    swiglu ? few_tiles<float, false, MOE_ACT_SWIGLU>(a, s) : few_tiles<float, false, MOE_ACT_SILU>(a, s);
  return hipGetLastError();
}

}  // namespace moe
