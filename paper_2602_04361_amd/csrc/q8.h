// Codes and scales of the 8-bit cache: e4m3 (bias 7, largest value 448) with E8M0
// exponent bytes, one a block of tokens and head.
#pragma once

#include "device_common.h"
#include "launch.h"

namespace sparvar {

constexpr float kE4m3Max = 448.f;  // 1.75 * 2^8
constexpr int kScaleExpMin = -100, kScaleExpMax = 112;

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;

// Smallest e with top <= 448 * 2^e, clamped (top >= 0). With top = m * 2^x, 1 <= m < 2:
// x - 8 where m <= 1.75, x - 7 otherwise, so it is read off the bits, exactly.
__device__ __forceinline__ int32_t block_exponent(float top) {
  const uint32_t b = __float_as_uint(top);
  const int32_t e = (int32_t)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
  return e < kScaleExpMin ? kScaleExpMin : (e > kScaleExpMax ? kScaleExpMax : e);
}

// 2^e as a float, for an E8M0 byte (e + 127) in 1..254.
__device__ __forceinline__ float scale_of_byte(uint32_t byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ float pow2f(int32_t e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Four codes of values within the format's range.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
#if defined(__HIP_DEVICE_COMPILE__)
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  return (uint32_t)w;
#else
  return 0;
#endif
}

// Four codes of x * inv (inv = 2^-e, so the product is exact but for underflow far below
// a code's step): rounded to nearest even, saturated at 448, NaN kept.
__device__ __forceinline__ uint32_t encode4(const float* x, float inv) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float t = x[i] * inv;
    const float s = fminf(fmaxf(t, -kE4m3Max), kE4m3Max);
    y[i] = t == t ? s : t;
  }
  return codes4(y[0], y[1], y[2], y[3]);
}

// Values of four codes times s.
__device__ __forceinline__ void decode4(uint32_t w, float s, float* x) {
#if defined(__HIP_DEVICE_COMPILE__)
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  x[0] = a[0] * s;
  x[1] = a[1] * s;
  x[2] = b[0] * s;
  x[3] = b[1] * s;
#endif
}

// Two words of four bf16 values: the codes times s, exact (4 significant bits).
__device__ __forceinline__ void decode4_bf16(uint32_t w, float s, uint32_t& lo, uint32_t& hi) {
#if defined(__HIP_DEVICE_COMPILE__)
  lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, s, false));
  hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, s, true));
#endif
}

}  // namespace sparvar
