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

// Query fragments for the products with K's codes: the row divided by a power of two (its
// largest magnitude then in (224, 448]) as the sum of two e4m3 values. bf16 has 8 significant
// bits and e4m3 4. What the larger part leaves is at most 16, so the smaller one is stored
// times 2^4, under a scale byte of its own: its last place is 2^-13. The sum is the query itself
// for elements from 2^-6 on, among them all from 2^-13 of the row's largest; below, it is off by
// at most half that place, 2^-14 / 224 < 2^-21 of the largest. Rows of one channel of 100 beside
// normals times 0.1, keys of normals times 4: the split alone, in exact sums, moves the LSE by
// 3e-5 (without the 2^4 by 2e-3). The rate is that of one bf16 product (two e4m3 ones at twice
// its rate), and K needs no conversion. Step t of a half covers channels 64 t + 32 half .. + 32,
// as K fragments of 8-bit codes do, or (MIXED: beside 4-bit codes, whose lanes hold the 32 channels of
// one half in a row) the 16 from 64 t + 16 half on and the 16 from 32 further, where the instruction
// looks for an 8-bit operand's.
typedef __attribute__((ext_vector_type(8))) int i32x8;

template <int D, bool MIXED = false>
struct QFragF8 {
  i32x8 hi[D / 64], lo[D / 64];
  int32_t scale;  // E8M0 bytes: of hi, and above it of lo
  __device__ __forceinline__ void load(const bf16_bits* row, int half) {
    u32x4 raw[D / 16];
    float top = 0.f;
#pragma unroll
    for (int t = 0; t < D / 64; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        raw[4 * t + i] = ldg16(row + 64 * t + (MIXED ? 16 * half + 8 * i + 16 * (i >> 1) : 32 * half + 8 * i));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          top = fmaxf(top, fabsf(__uint_as_float(raw[4 * t + i][e] << 16)));
          top = fmaxf(top, fabsf(__uint_as_float(raw[4 * t + i][e] & 0xffff0000u)));
        }
      }
    const int32_t e2 = block_exponent(max_halves(top));
    const float inv = pow2f(-e2);
    scale = (e2 + 127) | (e2 + 123) << 8;
#pragma unroll
    for (int t = 0; t < D / 64; ++t)
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        const uint32_t a = raw[4 * t + w / 2][2 * (w & 1)], b = raw[4 * t + w / 2][2 * (w & 1) + 1];
        const float x[4] = {__uint_as_float(a << 16) * inv, __uint_as_float(a & 0xffff0000u) * inv,
                            __uint_as_float(b << 16) * inv, __uint_as_float(b & 0xffff0000u) * inv};
        const uint32_t h = codes4(x[0], x[1], x[2], x[3]);
        float y[4];
        decode4(h, 1.f, y);
        hi[t][w] = (int)h;
        lo[t][w] = (int)codes4((x[0] - y[0]) * 16.f, (x[1] - y[1]) * 16.f, (x[2] - y[2]) * 16.f, (x[3] - y[3]) * 16.f);
      }
  }
};

}  // namespace sparvar
