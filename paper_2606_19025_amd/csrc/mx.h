// MXFP4 (microscaled 4-bit floats) on the device: blocks of 32 consecutive values of a row
// share an E8M0 scale 2^(s - 127); each value is an E2M1 code (sign, two exponent bits, one
// mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6).
#pragma once
#include "common.h"

namespace moe {

constexpr int MX_BLOCK = 32;
// Bytes of a row of scales: whole words, so that four blocks' scales load as one.
__host__ __device__ inline int mx_stride(int cols) { return (cols + 127) / 128 * 4; }

// The scale code of a block from the bits of its largest magnitude: floor(log2) - 2 puts
// that magnitude in [4, 8), of which values past 6 saturate.  255 (NaN) where the block
// holds an infinity or a NaN.
DEVI unsigned mx_scale_code(unsigned top_bits) {
  const int e = (int)(top_bits >> 23);  // (biased as E8M0 is)
  return e == 255 ? 255u : (unsigned)(e > 2 ? e - 2 : 0);
}

// Eight values to codes (value i in nibble i) under scale code s, rounded to nearest even.
// The instruction reads the scale from the exponent bits of an fp32 value; scales near the
// smallest one are moved up with their values (exactly), away from its edge.
DEVI unsigned mx_codes8(const float* v, unsigned s) {
  float a[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] = v[i];
  if (s < 64) {
    s += 64;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] *= 0x1p64f;
  }
  const float scale = __uint_as_float(s << 23);
  unsigned c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, a[0], a[1], scale, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, a[2], a[3], scale, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, a[4], a[5], scale, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, a[6], a[7], scale, 3);
  return s == 255 ? 0u : c;
}

// 2^(s - 127) as fp32: a subnormal for s = 0, NaN for 255.
DEVI float mx_scale_f32(unsigned s) {
  return __uint_as_float(s == 0 ? 0x00400000u : s == 255 ? 0x7fc00000u : s << 23);
}

typedef float f32x2_v __attribute__((ext_vector_type(2)));
// The eight values of a word of codes under scale 1 times `scale`.
DEVI void mx_values8(unsigned c, float scale, float* out) {
  const f32x2_v v0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0);
  const f32x2_v v1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 1);
  const f32x2_v v2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 2);
  const f32x2_v v3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 3);
  const float v[8] = {v0[0], v0[1], v1[0], v1[1], v2[0], v2[1], v3[0], v3[1]};
#pragma unroll
  for (int i = 0; i < 8; ++i) out[i] = v[i] * scale;
}

}  // namespace moe
