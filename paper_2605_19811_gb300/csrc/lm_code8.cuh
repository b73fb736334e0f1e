// 8-bit codes with one power-of-two scale for each group of 128 channels of a
// row (the format is stated at lm_checkpoint8 in lionmuon.h): scale of a
// group from its largest magnitude, codes from values, values from codes.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <stdint.h>

#include "lionmuon.h"

namespace lm {
namespace code8 {
namespace {

// |x| as an integer that orders like the magnitude, with NaN above infinity.
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// Scale of a group whose largest magnitude has these bits: 2^e with the least
// e such that max <= limit 2^e.  With max = 2^(E-127) (1 + F 2^-23) and
// limit = 127 = 2^6 * 1.984375 (448 = 2^8 * 1.75), e = E - 127 - 6 (- 8), one
// more where the fraction F is beyond the limit's.  NaN for a group that holds
// a NaN or an infinity.
template <int kFormat>
__device__ __forceinline__ float group_scale(uint32_t max_bits) {
  if (max_bits >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
  const int E = (int)(max_bits >> 23);
  const uint32_t F = max_bits & 0x7FFFFFu;
  int e = kFormat == LM_CODE_I8 ? E - 6 + (F > 0x7E0000u ? 1 : 0) : E - 8 + (F > 0x600000u ? 1 : 0);
  e = max(e, kFormat == LM_CODE_I8 ? 1 : 10);   // biased: 2^-126, 2^-117
  return __uint_as_float((uint32_t)e << 23);
}
// 1 / scale (exact: a power of two); 0 for a NaN scale, whose codes are all 0.
__device__ __forceinline__ float inverse_scale(float s) {
  return s == s ? __uint_as_float((254u << 23) - __float_as_uint(s)) : 0.f;
}
// Two codes, the first in the low byte.
template <int kFormat>
__device__ __forceinline__ uint32_t encode2(float a, float b, float inv) {
  if (inv == 0.f) return 0u;   // 0 * infinity would be NaN
  a *= inv;
  b *= inv;
  // under the largest scale, 2^122 (2^120), the code 64 (256) would stand for 2^128
  constexpr float kCap = kFormat == LM_CODE_I8 ? 63.f : 240.f;
  if (inv == __uint_as_float(kFormat == LM_CODE_I8 ? 5u << 23 : 7u << 23)) {
    a = fminf(fmaxf(a, -kCap), kCap);
    b = fminf(fmaxf(b, -kCap), kCap);
  }
  if (kFormat == LM_CODE_I8) {
    // 1.5 2^23 + a rounds a to an integer (nearest even); its low byte is the code
    constexpr float kRound = 12582912.f;
    return __byte_perm(__float_as_uint(a + kRound), __float_as_uint(b + kRound), 0x0040) & 0xFFFFu;
  }
  return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}
// The values of the two codes in the low half of `two`, before the scale.
template <int kFormat>
__device__ __forceinline__ float2 decode2(uint32_t two) {
  if (kFormat == LM_CODE_I8)
    return make_float2((float)(int8_t)(two & 0xFFu), (float)(int8_t)((two >> 8) & 0xFFu));
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(two & 0xFFFFu), __NV_E4M3);
  return __half22float2(__half2(h));
}

}  // namespace
}  // namespace code8
}  // namespace lm
