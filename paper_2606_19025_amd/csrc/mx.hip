// To MXFP4 and back, row by row (the format: mx.h).
//
// Bound by HBM.  A lane takes 8 consecutive values, so that its 16 (fp32: 32) bytes load
// whole and its codes are one 4-byte word; the four lanes of a block share their largest
// magnitude, compared as bits (a NaN's are above infinity's).
//
// Measured: 45056 x 2048 bf16 to MXFP4 60 us, back 35 us (3.9 and 6.7 TB/s of both sides).
#include "kernels.h"
#include "mx.h"
#include "timing.h"

namespace moe {
namespace {

constexpr int MX_THREADS = 256;
constexpr int MX_UNITS = 4;  // words per lane

// 8 values of x, their fp32 bits
DEVI void load8(const float* p, float* v) {
  load16_f32(p, v);
  load16_f32(p + 4, v + 4);
}
DEVI void load8(const bf16_t* p, float* v) { load16_f32(p, v); }
DEVI void store8(float* p, const float* v) {
  store16_f32(p, v);
  store16_f32(p + 4, v + 4);
}
DEVI void store8(bf16_t* p, const float* v) { store16_f32(p, v); }

struct MxArgs {
  int64_t units;         // words of codes: rows * cols / 8
  uint64_t per_row_inv;  // ceil(2^64 / per_row)
  int per_row, stride;   // words of codes, bytes of scales of a row
  const int32_t* n_rows;
};

// Units to convert: those of the first *n_rows rows where that is given.
DEVI int64_t unit_end(const MxArgs& a) {
  if (!a.n_rows) return a.units;
  const int64_t n = *a.n_rows;
  return n <= 0 ? 0 : min(a.units, n * a.per_row);
}

// The unit's row, by a multiplication: exact while units * per_row < 2^64, which
// every tensor that fits in memory is far below.
DEVI int64_t row_of(const MxArgs& a, int64_t u) { return (int64_t)__umul64hi((uint64_t)u, a.per_row_inv); }

template <class E>
__global__ __launch_bounds__(MX_THREADS) void mx_quantize_kernel(const E* x, uint8_t* codes,
                                                                 uint8_t* scales, MxArgs a) {
  const int64_t end = unit_end(a);
  const int64_t u0 = (int64_t)blockIdx.x * (MX_THREADS * MX_UNITS) + threadIdx.x;
  if (u0 - threadIdx.x >= end) return;
  float v[MX_UNITS][8];
#pragma unroll
  for (int i = 0; i < MX_UNITS; ++i) {
    const int64_t u = u0 + i * MX_THREADS;
    if (u < end) load8(x + u * 8, v[i]);
  }
#pragma unroll
  for (int i = 0; i < MX_UNITS; ++i) {
    const int64_t u = u0 + i * MX_THREADS;
    if (u >= end) break;  // (whole blocks of four lanes: rows are whole blocks)
    unsigned top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[i][j]) & 0x7fffffffu);
    top = max(top, (unsigned)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xF, 0xF, false));
    top = max(top, (unsigned)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xF, 0xF, false));
    const unsigned s = mx_scale_code(top);
    const unsigned c = mx_codes8(v[i], s);
    *reinterpret_cast<unsigned*>(codes + u * 4) = c;
    if ((threadIdx.x & 3) == 0) {
      const int64_t row = row_of(a, u);
      const int b = (int)(u - row * a.per_row) >> 2;
      uint8_t* out = scales + row * a.stride;
      out[b] = (uint8_t)s;
      // the bytes past the last block are zero
      if (b == (a.per_row >> 2) - 1)
        for (int q = b + 1; q < a.stride; ++q) out[q] = 0;
    }
  }
}

template <class E>
__global__ __launch_bounds__(MX_THREADS) void mx_dequantize_kernel(const uint8_t* codes,
                                                                   const uint8_t* scales, E* x,
                                                                   MxArgs a) {
  const int64_t end = unit_end(a);
  const int64_t u0 = (int64_t)blockIdx.x * (MX_THREADS * MX_UNITS) + threadIdx.x;
  if (u0 - threadIdx.x >= end) return;
  unsigned c[MX_UNITS], s[MX_UNITS];
#pragma unroll
  for (int i = 0; i < MX_UNITS; ++i) {
    const int64_t u = u0 + i * MX_THREADS;
    if (u < end) {
      const int64_t row = row_of(a, u);
      c[i] = *reinterpret_cast<const unsigned*>(codes + u * 4);
      s[i] = scales[row * a.stride + ((u - row * a.per_row) >> 2)];
    }
  }
#pragma unroll
  for (int i = 0; i < MX_UNITS; ++i) {
    const int64_t u = u0 + i * MX_THREADS;
    if (u < end) {
      float v[8];
      mx_values8(c[i], mx_scale_f32(s[i]), v);
      store8(x + u * 8, v);
    }
  }
}

static_assert((kMxWords / (MX_THREADS * MX_UNITS) + 1) * MX_THREADS <= int64_t(1) << 32, "a grid holds every word");

MxArgs mx_args(int rows, int cols, const int32_t* n_rows) {
  MxArgs a;
  a.per_row = cols / 8;
  a.units = (int64_t)rows * a.per_row;
  a.per_row_inv = UINT64_MAX / (uint64_t)a.per_row + 1;  // ceil(2^64 / per_row)
  a.stride = mx_stride(cols);
  a.n_rows = n_rows;
  return a;
}

unsigned mx_blocks(const MxArgs& a) {
  return (unsigned)((a.units + MX_THREADS * MX_UNITS - 1) / (MX_THREADS * MX_UNITS));
}

}  // namespace

hipError_t launch_mx_quantize(const void* x, int bf16, int rows, int cols, const int32_t* n_rows,
                              uint8_t* codes, uint8_t* scales, hipStream_t s) {
  if (rows == 0) return hipSuccess;
  const MxArgs a = mx_args(rows, cols, n_rows);
  if (bf16)
    MOE_TIMED("mx_quantize", s, mx_quantize_kernel<<<mx_blocks(a), MX_THREADS, 0, s>>>(
                                    static_cast<const bf16_t*>(x), codes, scales, a));
  else
    MOE_TIMED("mx_quantize", s, mx_quantize_kernel<<<mx_blocks(a), MX_THREADS, 0, s>>>(
                                    static_cast<const float*>(x), codes, scales, a));
  return hipGetLastError();
}

hipError_t launch_mx_dequantize(const uint8_t* codes, const uint8_t* scales, int bf16, int rows,
                                int cols, const int32_t* n_rows, void* x, hipStream_t s) {
  if (rows == 0) return hipSuccess;
  const MxArgs a = mx_args(rows, cols, n_rows);
  if (bf16)
    MOE_TIMED("mx_dequantize", s, mx_dequantize_kernel<<<mx_blocks(a), MX_THREADS, 0, s>>>(
                                      codes, scales, static_cast<bf16_t*>(x), a));
  else
    MOE_TIMED("mx_dequantize", s, mx_dequantize_kernel<<<mx_blocks(a), MX_THREADS, 0, s>>>(
                                      codes, scales, static_cast<float*>(x), a));
  return hipGetLastError();
}

}  // namespace moe
