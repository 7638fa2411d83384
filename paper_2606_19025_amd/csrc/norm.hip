// Layer norm over rows of d elements: the pre-norm of the MoE layer.
//
//   mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps), xh = (x - mu) r
//   y  = xh w + b
//   backward, g = dy w:  dx = dres + r (g - mean(g) - xh mean(g xh))
//                        dw = sum_t dy xh,  db = sum_t dy
//
// Bound by HBM: each row is read once and kept in registers as fp32, so the
// variance is the mean of squared distances from the mean (no E[x^2] - mu^2,
// which cancels for rows far from zero).  A row belongs to one wave, or to the 4 or
// 16 waves of a block where rows are few or long (row_waves_fwd, row_waves_bwd).
//
// The backward sums dw and db over the rows that a block takes in registers and
// stores one fp32 partial row per block; a second launch adds the partials in
// block order, so the results do not depend on timing.
//
// Measured (bf16): 8192 x 2048 forward 15 us (4.5 TB/s), backward with dres 26 us (5.2), dw and
// db 4.7 us; 16384 x 4096 backward 100 us (5.4 TB/s).  One row: 2.6 us.  Rows of sixteen waves:
// 8192 x 8192 backward 125 us, 8192 x 16384 238 us (4.3 and 4.5 TB/s; they have 128 registers a lane, of
// which 3 to 17 are spilled, fetch nothing ahead and read w for every row).
#include "common.h"
#include "kernels.h"
#include "timing.h"

namespace moe {
namespace {

// Waves of a block whose rows take W waves each.
constexpr int block_waves(int W) { return W == 1 ? 4 : W; }
constexpr int kDwThreads = 1024;

struct NormArgs {
  const void* x;
  const float* w;
  const float* b;
  void* y;       // backward: dx
  float* mean;
  float* rstd;
  const void* dy;
  const void* dres;
  float* part;   // backward: [blocks][2][d]
  int T, d;
  float eps, inv_d;
};

// Sums of N values over the W waves of a row, in all their lanes.  buf: W > 1,
// two alternating rows of the block's partial sums (so that one barrier per row
// is enough: a row's writes are two barriers after the last reads of its buffer).
template <int W, int N>
DEVI void row_sums(float (&v)[N], float (*buf)[W], int& flip) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], o, 64);
  if constexpr (W > 1) {
    float (*p)[W] = buf + flip * N;
    flip ^= 1;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) p[i][threadIdx.x >> 6] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = p[i][0];
#pragma unroll
      for (int q = 1; q < W; ++q) v[i] += p[i][q];
    }
  }
}

// The lane's NV 16-byte vectors of a row: vector i is at element col(i).
template <class E, int W, int NV>
struct Row {
  static constexpr int VE = Vec16<E>::N;
  static constexpr int TPR = 64 * W;  // threads per row
  DEVI static int col(int i) { return ((int)threadIdx.x % TPR + i * TPR) * VE; }
  DEVI static void load(const void* p, size_t row, int d, u32x4_t (&v)[NV]) {
    const E* q = static_cast<const E*>(p) + row * d;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      v[i] = col(i) < d ? *reinterpret_cast<const u32x4_t*>(q + col(i)) : u32x4_t{0u, 0u, 0u, 0u};
  }
  DEVI static void unpack(const u32x4_t& v, float* out) {
    if constexpr (VE == 8) {
      const bf16x8_t b = __builtin_bit_cast(bf16x8_t, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) out[j] = (float)b[j];
    } else {
      const f32x4_t f = __builtin_bit_cast(f32x4_t, v);
#pragma unroll
      for (int j = 0; j < 4; ++j) out[j] = f[j];
    }
  }
  DEVI static void load_f32(const float* p, int c, float* out) {
#pragma unroll
    for (int j = 0; j < VE; j += 4) load16_f32(p + c + j, out + j);
  }
};

template <class E, int W, int NV>
__global__ __launch_bounds__(64 * block_waves(W)) void norm_fwd_kernel(NormArgs a) {
  using R = Row<E, W, NV>;
  constexpr int VE = R::VE;
  __shared__ float buf[2][W];
  const int t = blockIdx.x * (block_waves(W) / W) + (int)threadIdx.x / R::TPR;
  if (W == 1 && t >= a.T) return;  // (W > 1: the grid has one block per row)
  u32x4_t raw[NV];
  R::load(a.x, t, a.d, raw);
  float v[NV][VE];
  float s[1] = {0.f};
  int flip = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    R::unpack(raw[i], v[i]);
#pragma unroll
    for (int j = 0; j < VE; ++j) s[0] += v[i][j];
  }
  row_sums<W>(s, buf, flip);
  const float mu = s[0] * a.inv_d;
  s[0] = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (R::col(i) < a.d)
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        v[i][j] -= mu;
        s[0] += v[i][j] * v[i][j];
      }
  row_sums<W>(s, buf, flip);
  const float r = 1.0f / sqrtf(s[0] * a.inv_d + a.eps);
  if (threadIdx.x % R::TPR == 0) {
    a.mean[t] = mu;
    a.rstd[t] = r;
  }
  E* y = static_cast<E*>(a.y) + (size_t)t * a.d;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = R::col(i);
    if (c < a.d) {
      float w[VE], b[VE];
      R::load_f32(a.w, c, w);
      if (a.b) R::load_f32(a.b, c, b);
#pragma unroll
      for (int j = 0; j < VE; ++j) v[i][j] = v[i][j] * r * w[j] + (a.b ? b[j] : 0.f);
      store16_f32(y + c, v[i]);
    }
  }
}

// Blocks take rows in turn (a row per wave, or one per block).  A row's loads are issued
// before the previous row's arithmetic.
template <class E, int W, int NV, bool RES>
__global__ __launch_bounds__(64 * block_waves(W)) void norm_bwd_kernel(NormArgs a) {
  using R = Row<E, W, NV>;
  constexpr int VE = R::VE, ROWS = block_waves(W) / W;
  __shared__ float buf[4][W];
  extern __shared__ float cols[];  // [2][d], W == 1
  const int step = gridDim.x * ROWS;
  // sixteen waves leave a lane 128 registers: w is read again for each row (L1), and
  // the next row is not fetched ahead
  constexpr bool AHEAD = W < 16;
  float dw[NV][VE], db[NV][VE], w[NV][VE];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < VE; ++j) dw[i][j] = db[i][j] = w[i][j] = 0.f;
  auto load_w = [&]() {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (R::col(i) < a.d) R::load_f32(a.w, R::col(i), w[i]);
  };
  if (AHEAD) load_w();
  u32x4_t nx[NV], ny[NV], nr[RES ? NV : 1];
  float nmu = 0.f, nrs = 0.f;
  auto fetch = [&](int t) {
    R::load(a.x, t, a.d, nx);
    R::load(a.dy, t, a.d, ny);
    if constexpr (RES) R::load(a.dres, t, a.d, nr);
    nmu = a.mean[t];
    nrs = a.rstd[t];
  };
  int flip = 0;
  int t = blockIdx.x * ROWS + (int)threadIdx.x / R::TPR;
  if (AHEAD && t < a.T) fetch(t);
  for (; t < a.T; t += step) {  // (W > 1: the same rows in all of the block)
    if (!AHEAD) {
      fetch(t);
      load_w();
    }
    float xh[NV][VE], g[NV][VE], res[RES ? NV : 1][VE];
    const float mu = nmu, r = nrs;
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      R::unpack(nx[i], xh[i]);
      R::unpack(ny[i], g[i]);
      if constexpr (RES) R::unpack(nr[i], res[i]);
    }
    if (AHEAD && t + step < a.T) fetch(t + step);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      // past the row's end x, dy and w are zeros, and the mean is taken as zero: every sum is
      const float m = R::col(i) < a.d ? mu : 0.f;
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        xh[i][j] = (xh[i][j] - m) * r;
        dw[i][j] += g[i][j] * xh[i][j];
        db[i][j] += g[i][j];
        g[i][j] *= w[i][j];
        s[0] += g[i][j];
        s[1] += g[i][j] * xh[i][j];
      }
    }
    row_sums<W>(s, buf, flip);
    const float m0 = s[0] * a.inv_d, m1 = s[1] * a.inv_d;
    E* dx = static_cast<E*>(a.y) + (size_t)t * a.d;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = R::col(i);
      if (c < a.d) {
#pragma unroll
        for (int j = 0; j < VE; ++j) {
          g[i][j] = r * (g[i][j] - m0 - xh[i][j] * m1);
          if constexpr (RES) g[i][j] += res[i][j];
        }
        store16_f32(dx + c, g[i]);
      }
    }
  }
  // the block's partial row: with a row per wave the waves' sums are added in
  // wave order through LDS
  float* part = a.part + (size_t)blockIdx.x * 2 * a.d;
  if constexpr (W == 1) {
    for (int q = 0; q < ROWS; ++q) {
      if ((int)(threadIdx.x >> 6) == q)
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int c = R::col(i);
          if (c < a.d)
#pragma unroll
            for (int j = 0; j < VE; ++j) {
              cols[c + j] = (q ? cols[c + j] : 0.f) + dw[i][j];
              cols[a.d + c + j] = (q ? cols[a.d + c + j] : 0.f) + db[i][j];
            }
        }
      __syncthreads();
    }
    for (int c = threadIdx.x * 4; c < 2 * a.d; c += 64 * ROWS * 4)
      *reinterpret_cast<f32x4_t*>(part + c) = *reinterpret_cast<const f32x4_t*>(cols + c);
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = R::col(i);
      if (c < a.d)
#pragma unroll
        for (int j = 0; j < VE; j += 4) {
          *reinterpret_cast<f32x4_t*>(part + c + j) =
              f32x4_t{dw[i][j], dw[i][j + 1], dw[i][j + 2], dw[i][j + 3]};
          *reinterpret_cast<f32x4_t*>(part + a.d + c + j) =
              f32x4_t{db[i][j], db[i][j + 1], db[i][j + 2], db[i][j + 3]};
        }
    }
  }
}

// dw and db from the n partial rows [n][2][d]: a block takes 64 of the 2 d columns, sixteen
// threads (16 bytes each) by 64 shares of the partials, whose sums are added eight at a time.
// (Sixteen shares: 512 partials took 7 us, a thread's 32 loads one after another; now 4.)
__global__ __launch_bounds__(kDwThreads) void norm_dw_kernel(const float* part, int n, int d, float* dw,
                                                             float* db, int accumulate) {
  constexpr int P = kDwThreads / 16, G = 8;
  __shared__ f32x4_t sum[P][16];
  const int q = threadIdx.x & 15, p = threadIdx.x >> 4;
  const int c = (blockIdx.x * 16 + q) * 4;
  f32x4_t s = {0.f, 0.f, 0.f, 0.f};
  if (c < 2 * d)
    for (int i = p; i < n; i += P) s += *reinterpret_cast<const f32x4_t*>(part + (size_t)i * 2 * d + c);
  sum[p][q] = s;
  __syncthreads();
  if (p < G) {
    for (int i = p + G; i < P; i += G) s += sum[i][q];
    sum[p][q] = s;  // (read by this thread alone so far)
  }
  __syncthreads();
  if (p == 0 && c < 2 * d) {
    for (int i = 1; i < G; ++i) s += sum[i][q];
    float* out = c < d ? dw + c : db ? db + (c - d) : nullptr;
    if (out) {
      f32x4_t* o = reinterpret_cast<f32x4_t*>(out);
      *o = accumulate ? *o + s : s;
    }
  }
}

// Vectors per lane of a row of d elements shared by `waves` waves, as a power of two.
int vectors(int d, int ve, int waves) {
  int nv = 1;
  while (nv * 64 * waves * ve < d) nv *= 2;
  return nv;
}

// Waves per row: one where the rows are many and a lane then holds at most `one`
// vectors, else the fewest of 4 and 16 that leave a lane at most `more`.  Measured (us, one wave /
// four; launch included):
//   bf16      forward, d = 512   1024         2048         backward, d = 512   1024
//   1024      6.5 / 6.3          6.4 / 6.4    6.6 / 6.7    7.7 / 7.9    10.8 / 8.8
//   2048      6.6 / 6.9          6.5 / 6.8    8.2 / 7.5    8.3 / 8.6    12.2 / 10.1
//   4096      6.9 / 8.0          7.3 / 9.2    11.3 / 11.0  9.9 / 12.1   14.2 / 13.5
//   6144      6.9 / 10.0         8.9 / 11.4   13.6 / 14.3  10.8 / 16.1  15.7 / 16.2
//   8192      7.6 / 11.7         10.3 / 13.8  15.4 / 16.7  11.8 / 19.0  16.5 / 20.2
//   fp32      forward, d = 512   1024         backward, d = 512   640          768          896          1024
//   1024      6.5 / 6.4          6.7 / 6.8    7.9 / 7.4                                                  10.6 / 8.4
//   2048      7.0 / 6.6          7.1 / 7.3    8.6 / 8.4                                                  12.7 / 9.8
//   4096      7.4 / 8.6          10.0 / 10.3  10.0 / 11.2  12.0 / 11.9  12.7 / 12.3  14.2 / 12.7  14.5 / 13.8
//   6144      8.1 / 10.9         11.7 / 13.2  11.2 / 14.8  14.0 / 16.2  15.9 / 15.9  17.7 / 16.2  19.1 / 16.9
//   8192      9.3 / 12.7         13.8 / 15.9  13.2 / 17.9  16.8 / 19.0  18.7 / 19.2  21.0 / 20.6  22.5 / 21.5
//   16384     15.2 / 20.1        24.3 / 26.5  20.9 / 28.8  25.8 / 31.0  29.1 / 30.9  33.0 / 33.1  37.0 / 37.1
int row_waves(int T, int d, int ve, int one, int more) {
  if (T >= 4096 && vectors(d, ve, 1) <= one) return 1;
  return vectors(d, ve, 4) <= more ? 4 : 16;
}
int row_waves_fwd(int T, int d, int ve) { return row_waves(T, d, ve, 4, 4); }
// (a lane of the backward holds six fp32 values per element: 16 elements at most; fp32 rows past
// 768 columns take four waves)
int row_waves_bwd(int T, int d, int ve) {
  return row_waves(T, d, ve, ve == 4 && d > 768 ? 2 : 16 / ve, 16 / ve);
}

// Blocks of the backward: each writes a partial row of 2 d, so that past one per CU a block
// takes at least four rows (1024 rows, d = 4096: 256 blocks 12.7 us, 512 14.5), up to two per
// CU (8192 rows: 256 blocks 43 us, 512 38, 1024 43).
int bwd_blocks(int T, int d, int ve) {
  const int W = row_waves_bwd(T, d, ve), units = ceil_div(T, block_waves(W) / W);
  return std::min(std::max(std::min(units, num_cus()), ceil_div(T, 4)), std::min(units, 2 * num_cus()));
}

// Rows of one launch: a grid dimension holds less than 2^32 threads (a larger one is not refused
// but taken modulo 2^32), so that more rows are taken by several launches.  A power of two.
constexpr int rows_per_launch(int W) { return (int)((int64_t(1) << 31) / (64 * W)); }

template <class E>
void fwd_rows(const NormArgs& a, int W, hipStream_t s) {
  constexpr int VE = Vec16<E>::N;
  const int nv = vectors(a.d, VE, W);
#define NORM_FWD(W_, NV_)                                                                 \
  MOE_TIMED("norm_fwd", s, norm_fwd_kernel<E, W_, NV_>                                    \
            <<<ceil_div(a.T, block_waves(W_) / W_), 64 * block_waves(W_), 0, s>>>(a))
  if (W == 1) {
    if (nv == 1) NORM_FWD(1, 1);
    else if (nv == 2) NORM_FWD(1, 2);
    else NORM_FWD(1, 4);
  } else if (W == 4) {
    if (nv == 1) NORM_FWD(4, 1);
    else if (nv == 2) NORM_FWD(4, 2);
    else NORM_FWD(4, 4);
  } else {
    // (past four waves' reach a lane holds at least half of its sixteen elements)
    if constexpr (VE == 8) NORM_FWD(16, 2);
    else NORM_FWD(16, 4);
  }
#undef NORM_FWD
}

template <class E>
hipError_t fwd(const NormArgs& a, hipStream_t s) {
  const int W = row_waves_fwd(a.T, a.d, Vec16<E>::N), most = rows_per_launch(W);
  for (int t = 0; t < a.T; t += most) {
    NormArgs part = a;
    part.x = static_cast<const E*>(a.x) + (size_t)t * a.d;
    part.y = static_cast<E*>(a.y) + (size_t)t * a.d;
    part.mean = a.mean + t;
    part.rstd = a.rstd + t;
    part.T = std::min(a.T - t, most);
    fwd_rows<E>(part, W, s);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <class E, bool RES>
void bwd(const NormArgs& a, int blocks, hipStream_t s) {
  constexpr int VE = Vec16<E>::N;
  const int W = row_waves_bwd(a.T, a.d, VE), nv = vectors(a.d, VE, W);
  const size_t lds = W == 1 ? (size_t)2 * a.d * sizeof(float) : 0;
#define NORM_BWD(W_, NV_)                                  \
  MOE_TIMED("norm_bwd", s, norm_bwd_kernel<E, W_, NV_, RES> \
            <<<blocks, 64 * block_waves(W_), lds, s>>>(a))
  if (W == 1) {
    if (nv == 1) NORM_BWD(1, 1);
    else if (nv == 2) NORM_BWD(1, 2);
    else if constexpr (VE == 4) NORM_BWD(1, 4);
  } else if (W == 4) {
    if (nv == 1) NORM_BWD(4, 1);
    else if (nv == 2) NORM_BWD(4, 2);
    else if constexpr (VE == 4) NORM_BWD(4, 4);
  } else {
    NORM_BWD(16, 16 / VE);
  }
#undef NORM_BWD
}

}  // namespace

hipError_t launch_norm_fwd(const void* x, const float* w, const float* b, int bf16, int T, int d,
                           float eps, void* y, float* mean, float* rstd, hipStream_t s) {
  if (T == 0) return hipSuccess;
  NormArgs a{};
  a.x = x; a.w = w; a.b = b; a.y = y; a.mean = mean; a.rstd = rstd;
  a.T = T; a.d = d; a.eps = eps; a.inv_d = 1.0f / (float)d;
  return bf16 ? fwd<bf16_t>(a, s) : fwd<float>(a, s);
}

size_t norm_bwd_ws_bytes(int T, int d, int bf16) {
  return (size_t)bwd_blocks(T, d, bf16 ? 8 : 4) * 2 * d * sizeof(float);
}

hipError_t launch_norm_bwd(const void* dy, const void* x, const float* w, const float* mean,
                           const float* rstd, int bf16, int T, int d, const void* dres, void* dx,
                           float* dw, float* db, int accumulate, void* ws, hipStream_t s) {
  NormArgs a{};
  a.x = x; a.w = w; a.y = dx; a.dy = dy; a.dres = dres;
  a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
  a.part = static_cast<float*>(ws);
  a.T = T; a.d = d; a.inv_d = 1.0f / (float)d;
  const int blocks = bwd_blocks(T, d, bf16 ? 8 : 4);
  if (T > 0) {
    if (bf16) dres ? bwd<bf16_t, true>(a, blocks, s) : bwd<bf16_t, false>(a, blocks, s);
    else dres ? bwd<float, true>(a, blocks, s) : bwd<float, false>(a, blocks, s);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  MOE_TIMED("norm_dw", s,
            norm_dw_kernel<<<ceil_div(2 * d, 64), kDwThreads, 0, s>>>(a.part, blocks, d, dw, db, accumulate));
  return hipGetLastError();
}

}  // namespace moe
