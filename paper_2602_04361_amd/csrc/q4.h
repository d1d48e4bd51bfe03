// Codes and scales of the 4-bit cache: e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives; two
// a byte, the even channel low) with an E8M0 exponent byte a token and 32 channels.
#pragma once

#include "device_common.h"
#include "launch.h"

namespace sparvar {

constexpr int kQ4Group = 32;  // channels of a scale
constexpr int kQ4ExpMin = -100, kQ4ExpMax = 112;
constexpr uint32_t kQ4NaN = 255;  // scale byte of a group that held a NaN (no code stands for one)

typedef __attribute__((ext_vector_type(2))) __bf16 q4_bf16x2;
typedef __attribute__((ext_vector_type(2))) float q4_f32x2;

// Scale byte of a group: top is the largest of its values' bits without their signs, as whole numbers
// (a NaN's are above infinity's). e is the smallest with top <= 7 * 2^e: nothing below 7 is off by
// more than half the step of 2 that lies around it, so that 6 stands for up to 7. With top = m * 2^x,
// 1 <= m < 2: x - 2 where m <= 1.75, x - 1 otherwise.
__device__ __forceinline__ uint32_t q4_scale_byte(uint32_t top) {
  if (top > 0x7f800000u) return kQ4NaN;
  const int32_t e = (int32_t)(top >> 23) - 127 - 2 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (uint32_t)((e < kQ4ExpMin ? kQ4ExpMin : (e > kQ4ExpMax ? kQ4ExpMax : e)) + 127);
}

// The scale that a byte stands for, as the conversions take it: its exponent counts, and 255 makes
// their results NaN.
__device__ __forceinline__ float q4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight codes of x / scale: to nearest, ties to even, saturated at 6.
__device__ __forceinline__ uint32_t q4_encode8(const float (&x)[8], float scale) {
#if defined(__HIP_DEVICE_COMPILE__)
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
  return w;
#else
  return 0;
#endif
}

// Eight codes as bf16 values times scale, exact (two significant bits).
__device__ __forceinline__ u32x4 q4_decode8_bf16(uint32_t w, float scale) {
#if defined(__HIP_DEVICE_COMPILE__)
  u32x4 o;
  o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
  o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
  o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
  o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
  return o;
#else
  return u32x4{0, 0, 0, 0};
#endif
}

__device__ __forceinline__ void q4_decode8(uint32_t w, float scale, float (&x)[8]) {
#if defined(__HIP_DEVICE_COMPILE__)
  const q4_f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1),
                 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
  x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1];
  x[4] = c[0], x[5] = c[1], x[6] = d[0], x[7] = d[1];
#endif
}

}  // namespace sparvar
