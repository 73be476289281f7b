// The 8-bit cache's number format: e4m3 codes (4 exponent bits, bias 7, 3 mantissa bits, no infinities) times a scale per block of
// tokens and head.
#pragma once

#include "fkv_dpp.h"
#include "fkv_internal.h"

namespace fkv {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float floatx2;

constexpr float kScaleMin = 0x1p-126f;

__device__ __forceinline__ bool is_finite(float x) { return __builtin_fabsf(x) < __builtin_inff(); }

// The smallest power of two p >= 2^-126 with a <= 448 p, for finite a >= 0: 448 = 1.75 * 2^8, so it is a's exponent less 8, plus 1
// where the mantissa is over 1.75.  Whole numbers only: exact.
__device__ __forceinline__ float scale_for(float a) {
  const uint32_t u = __float_as_uint(a);
  const int e = (int)(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return __uint_as_float((uint32_t)max(e, 1) << 23);
}

// Codes of 8 values times `inv` (the reciprocal of a power of two: exact), rounded to nearest even; NaN for what is not finite.  The
// products are at most 448 in size, what the conversion makes of larger ones never shows.
__device__ __forceinline__ u32x2 encode8(const float *x, float inv) {
  u32x2 r;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = is_finite(x[4 * w + i]) ? x[4 * w + i] * inv : __uint_as_float(0x7FC00000u);
    int p = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    p = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], p, true);
    r[w] = (uint32_t)p;
  }
  return r;
}

// Codes of code * ratio, ratio <= 1: four at once.
__device__ __forceinline__ uint32_t rescale4(uint32_t codes, float ratio) {
  const floatx2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
  int p = __builtin_amdgcn_cvt_pk_fp8_f32(lo[0] * ratio, lo[1] * ratio, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(hi[0] * ratio, hi[1] * ratio, p, true);
}

__device__ __forceinline__ void unpack8(u32x4 v, float *x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(v[i] << 16);
    x[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ u32x4 pack8(const float *x) {  // rounded to nearest even
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_bit_cast(uint32_t, (bf16x2){(__bf16)x[2 * i], (__bf16)x[2 * i + 1]});
  return r;
}

}  // namespace fkv
