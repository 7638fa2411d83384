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

// mean and 1 / deviation of v (zeros past the row's end), which becomes v - mean
template <class R, int W, int NV>
DEVI void center(const BlockArgs& a, float (&v)[NV][R::VE], float (*buf)[W], int& flip, float& mu,
                 float& r) {
  float s[1] = {0.f};
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < R::VE; ++j) s[0] += v[i][j];
  row_sums<W>(s, buf, flip);
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
  row_sums<W>(s, buf, flip);
  r = 1.0f / sqrtf(s[0] * a.inv_d + a.p.eps);
}

template <class E, int W, int NV>
__global__ __launch_bounds__(64 * block_waves(W)) void block_norm_fwd_kernel(BlockArgs a) {
  using R = Row<E, W, NV>;
  constexpr int VE = R::VE;
  __shared__ float buf[2][W];
  const moe_block_norm& p = a.p;
  const int t = blockIdx.x * (block_waves(W) / W) + (int)threadIdx.x / R::TPR;
  if (W == 1 && t >= p.T) return;  // (W > 1: the grid has one block per row)
  const bool first = threadIdx.x % R::TPR == 0;
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

// Blocks take rows in turn (a row per wave, or one per block).  PRE, POST: the norms that there
// are.  A row's loads are issued before the previous row's arithmetic.
template <class E, int W, int NV, bool PRE, bool POST>
__global__ __launch_bounds__(64 * block_waves(W)) void block_norm_bwd_kernel(BlockArgs a) {
  using R = Row<E, W, NV>;
  constexpr int VE = R::VE, ROWS = block_waves(W) / W;
  __shared__ float buf[6][W];
  extern __shared__ float cols[];  // [4][d], W == 1
  const moe_block_norm& p = a.p;
  const bool channel = p.gate_kind == MOE_BLOCK_GATE_CHANNEL;
  const bool token = p.gate_kind == MOE_BLOCK_GATE_TOKEN;
  const int step = gridDim.x * ROWS;
  constexpr bool AHEAD = W < 16;
  float s[kSums][NV][VE];
#pragma unroll
  for (int q = 0; q < kSums; ++q)
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < VE; ++j) s[q][i][j] = 0.f;
  u32x4_t nu[PRE ? NV : 1], nx[PRE ? NV : 1], nf[NV], nr[NV];
  float n_mx = 0.f, n_rx = 0.f, n_mf = 0.f, n_rf = 0.f, n_g = 1.f;
  auto fetch = [&](int t) {
    if constexpr (PRE) {
      R::load(p.du, t, p.d, nu);
      R::load(p.x_out, t, p.d, nx);
      n_mx = p.pre_mean[t];
      n_rx = p.pre_rstd[t];
    }
    R::load(p.f, t, p.d, nf);
    if (p.dres) R::load(p.dres, t, p.d, nr);
    if constexpr (POST) {
      n_mf = p.post_mean[t];
      n_rf = p.post_rstd[t];
    }
    if (token) n_g = p.gate[t];
  };
  int flip = 0;
  int t = blockIdx.x * ROWS + (int)threadIdx.x / R::TPR;
  if (AHEAD && t < p.T) fetch(t);
  for (; t < p.T; t += step) {  // (W > 1: the same rows in all of the block)
    if (!AHEAD) fetch(t);
    float G[NV][VE], fh[NV][VE];
    const float mf = n_mf, rf = n_rf, ag = token ? p.scale * n_g : p.scale;
    // ---- the pre-norm's backward: G
    if constexpr (PRE) {
      float xh[NV][VE];
      const float mx = n_mx, rx = n_rx;
      float q[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        // past the row's end x, du and w are zeros, and the mean is taken as zero: every sum is
        const bool in = R::col(i) < p.d;
        const float m = in ? mx : 0.f;
        float w[VE] = {};
        if (in) R::load_f32(p.pre_weight, R::col(i), w);
        R::unpack(nx[i], xh[i]);
        R::unpack(nu[i], G[i]);
#pragma unroll
        for (int j = 0; j < VE; ++j) {
          xh[i][j] = (xh[i][j] - m) * rx;
          s[0][i][j] += G[i][j] * xh[i][j];
          s[1][i][j] += G[i][j];
          G[i][j] *= w[j];
          q[0] += G[i][j];
          q[1] += G[i][j] * xh[i][j];
        }
      }
      row_sums<W>(q, buf, flip);
      const float m0 = q[0] * a.inv_d, m1 = q[1] * a.inv_d;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const bool in = R::col(i) < p.d;
        float res[VE] = {};
        if (p.dres) R::unpack(nr[i], res);
#pragma unroll
        for (int j = 0; j < VE; ++j)
          G[i][j] = in ? res[j] + rx * (G[i][j] - m0 - xh[i][j] * m1) : 0.f;
      }
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i) R::unpack(nr[i], G[i]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) R::unpack(nf[i], fh[i]);
    if (AHEAD && t + step < p.T) fetch(t + step);
    {
      E* dx = static_cast<E*>(p.dx) + (size_t)t * p.d;
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (R::col(i) < p.d) store16_f32(dx + R::col(i), G[i]);
    }
    // ---- the gate and the post norm: G becomes dn (times w_post)
    float q[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = R::col(i);
      const bool in = c < p.d;
      float w[VE] = {}, b[VE] = {}, g[VE] = {};
      if (in) {
        if (POST) R::load_f32(p.post_weight, c, w);
        if (POST && p.post_bias) R::load_f32(p.post_bias, c, b);
        if (channel) R::load_f32(p.gate, c, g);
      }
      const float m = POST && in ? mf : 0.f;
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        if constexpr (POST) fh[i][j] = (fh[i][j] - m) * rf;
        if (token) q[2] += G[i][j] * (POST ? fh[i][j] * w[j] + b[j] : fh[i][j]);
        G[i][j] *= ag;
        s[2][i][j] += G[i][j] * fh[i][j];
        s[3][i][j] += G[i][j];
        if (channel) G[i][j] *= g[j];
        if constexpr (POST) {
          G[i][j] *= w[j];
          q[0] += G[i][j];
          q[1] += G[i][j] * fh[i][j];
        }
      }
    }
    if (POST || token) row_sums<W>(q, buf, flip);
    if (token && threadIdx.x % R::TPR == 0) p.d_gate[t] = p.scale * q[2];
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
  // the block's partial row: with a row per wave the waves' sums are added in
  // wave order through LDS
  float* part = a.part + (size_t)blockIdx.x * kSums * p.d;
  if constexpr (W == 1) {
    for (int q = 0; q < ROWS; ++q) {
      if ((int)(threadIdx.x >> 6) == q)
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int c = R::col(i);
          if (c < p.d)
#pragma unroll
            for (int k = 0; k < kSums; ++k)
#pragma unroll
              for (int j = 0; j < VE; ++j)
                cols[k * p.d + c + j] = (q ? cols[k * p.d + c + j] : 0.f) + s[k][i][j];
        }
      __syncthreads();
    }
    for (int c = threadIdx.x * 4; c < kSums * p.d; c += 64 * ROWS * 4)
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

// The weights' gradients from the n partial rows [n][4][d]: a block takes 16 columns, four
// threads (16 bytes each) by 128 shares of the partials for each sum in turn.
constexpr int kDwShares = 128;
__global__ __launch_bounds__(4 * kDwShares) void block_norm_dw_kernel(BlockArgs a, int n) {
  const moe_block_norm& p = a.p;
  __shared__ f32x4_t sum[kDwShares][4];
  __shared__ f32x4_t tot[kSums][4];
  const int q = threadIdx.x & 3, sh = threadIdx.x >> 2;
  const int c = (blockIdx.x * 4 + q) * 4;
  for (int k = 0; k < kSums; ++k) {
    f32x4_t s = {0.f, 0.f, 0.f, 0.f};
    if (c < p.d)
      for (int i = sh; i < n; i += kDwShares)
        s += *reinterpret_cast<const f32x4_t*>(a.part + ((size_t)i * kSums + k) * p.d + c);
    sum[sh][q] = s;
    __syncthreads();
    if (sh < 8) {
      for (int i = sh + 8; i < kDwShares; i += 8) s += sum[i][q];
      sum[sh][q] = s;  // (read by this thread alone so far)
    }
    __syncthreads();
    if (sh == 0) {
      for (int i = 1; i < 8; ++i) s += sum[i][q];
      tot[k][q] = s;
    }
    __syncthreads();
  }
  if (sh != 0 || c >= p.d) return;
  auto put = [&](float* out, f32x4_t v) {
    if (!out) return;
    f32x4_t* o = reinterpret_cast<f32x4_t*>(out + c);
    *o = p.accumulate ? *o + v : v;
  };
  const f32x4_t s3 = tot[2][q], s4 = tot[3][q];
  if (p.pre_weight) {
    put(p.d_pre_weight, tot[0][q]);
    put(p.d_pre_bias, tot[1][q]);
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

int waves_fwd(int T, int d, int ve) {
  if (T >= 4096 && vectors(d, ve, 1) <= 2) return 1;
  return vectors(d, ve, 4) <= 2 ? 4 : 16;
}
// (a lane of the backward holds four sums and four values per element)
int waves_bwd(int T, int d, int ve) {
  if (T >= 4096 && vectors(d, ve, 1) <= 8 / ve) return 1;
  return vectors(d, ve, 4) <= 16 / ve ? 4 : 16;
}

int blocks_bwd(int T, int d, int ve) {
  const int W = waves_bwd(T, d, ve), units = ceil_div(T, block_waves(W) / W);
  return std::min(std::max(std::min(units, num_cus()), ceil_div(T, 4)), std::min(units, 2 * num_cus()));
}

template <class E>
void fwd_rows(const BlockArgs& a, int W, hipStream_t s) {
  const int nv = vectors(a.p.d, Vec16<E>::N, W);
#define BLOCK_FWD(W_, NV_)                                                                \
  MOE_TIMED("block_norm_fwd", s, block_norm_fwd_kernel<E, W_, NV_>                        \
            <<<ceil_div(a.p.T, block_waves(W_) / W_), 64 * block_waves(W_), 0, s>>>(a))
  if (W == 1) {
    if (nv == 1) BLOCK_FWD(1, 1);
    else BLOCK_FWD(1, 2);
  } else if (W == 4) {
    if (nv == 1) BLOCK_FWD(4, 1);
    else BLOCK_FWD(4, 2);
  } else {
    if (nv == 1) BLOCK_FWD(16, 1);
    else if (nv == 2) BLOCK_FWD(16, 2);
    else if constexpr (Vec16<E>::N == 4) BLOCK_FWD(16, 4);
  }
#undef BLOCK_FWD
}

template <class E>
hipError_t fwd(const BlockArgs& a, hipStream_t s) {
  const moe_block_norm& p = a.p;
  const int W = waves_fwd(p.T, p.d, Vec16<E>::N), most = rows_per_launch(W);
  for (int t = 0; t < p.T; t += most) {
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
    fwd_rows<E>(part, W, s);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <class E, bool PRE, bool POST>
void bwd(const BlockArgs& a, int blocks, hipStream_t s) {
  constexpr int VE = Vec16<E>::N;
  const int d = a.p.d, W = waves_bwd(a.p.T, d, VE), nv = vectors(d, VE, W);
  const size_t lds = W == 1 ? (size_t)kSums * d * sizeof(float) : 0;
#define BLOCK_BWD(W_, NV_)                                                    \
  MOE_TIMED("block_norm_bwd", s, block_norm_bwd_kernel<E, W_, NV_, PRE, POST> \
            <<<blocks, 64 * block_waves(W_), lds, s>>>(a))
  if (W == 1) {
    if (nv == 1) BLOCK_BWD(1, 1);
    else if constexpr (VE == 4) BLOCK_BWD(1, 2);
  } else if (W == 4) {
    if (nv == 1) BLOCK_BWD(4, 1);
    else if (nv == 2) BLOCK_BWD(4, 2);
    else if constexpr (VE == 4) BLOCK_BWD(4, 4);
  } else {
    if (nv == 1) BLOCK_BWD(16, 1);
    else if (nv == 2) BLOCK_BWD(16, 2);
    else if constexpr (VE == 4) BLOCK_BWD(16, 4);
  }
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
            block_norm_dw_kernel<<<ceil_div(p->d, 16), 4 * kDwShares, 0, s>>>(a, blocks));
  return hipGetLastError();
}

}  // namespace moe
