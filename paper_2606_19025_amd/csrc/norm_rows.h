// Rows of activations in registers, shared by the row norms (norm.hip,
// block_norm.hip): a row belongs to one wave, or to the W waves of a block.
#pragma once
#include "common.h"

namespace moe {

// Waves of a block whose rows take W waves each.
constexpr int block_waves(int W) { return W == 1 ? 4 : W; }

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

// Vectors per lane of a row of d elements shared by `waves` waves, as a power of two.
inline int vectors(int d, int ve, int waves) {
  int nv = 1;
  while (nv * 64 * waves * ve < d) nv *= 2;
  return nv;
}

// Rows of one launch: a grid dimension holds less than 2^32 threads (a larger one is not refused
// but taken modulo 2^32), so that more rows are taken by several launches.  A power of two.
constexpr int rows_per_launch(int W) { return (int)((int64_t(1) << 31) / (64 * W)); }

}  // namespace moe
