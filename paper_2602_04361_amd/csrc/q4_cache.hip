// Rows of a cache to 4 bits and back. A row needs nothing but itself: a scale belongs to 32 of its
// channels. Both ways are copies by their cost: 2 to 4 bytes an element on one side, 0.53 on the other.
//
// A lane takes 8 channels (16 or 32 bytes of the row, 4 of the codes), so that four neighbouring
// lanes hold a scale's channels and find their largest magnitude by two exchanges. Four loads of a lane
// are in flight. 10521 tokens of 2 x 16 heads of 128, bf16, to codes and back: 55 and 32 us, 88 together among
// others' passes, 436 MB: 5.0 TB/s, a large copy's rate being 5.2. A row as small as a scale of 36 tokens costs its
// launch, 2.8 us.
#include "q4.h"

namespace sparvar {

namespace {

constexpr int kNT = 256;
constexpr int kUnits = 4;  // eights of a lane, a workgroup's width apart

__device__ __forceinline__ void load8(const bf16_bits* p, float (&x)[8]) {
  const u32x4 w = ldg16(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
  x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}

constexpr int kDppXor1 = 0xB1, kDppXor2 = 0x4E;  // lane ^ 1, lane ^ 2

struct QuantizeIO {
  const void *k, *v;
  int64_t bh_stride;
  Q4View c;
  int32_t units, first_unit, groups;  // eights of a plane's rows, and of the cache before them; workgroups a plane
};

template <class T>
__global__ __launch_bounds__(kNT) void kv_quantize_q4_kernel(QuantizeIO io) {
  const int32_t g = blockIdx.x % io.groups, rest = blockIdx.x / io.groups;
  const bool is_v = rest & 1;
  const int32_t plane = rest >> 1;
  const T* src = static_cast<const T*>(is_v ? io.v : io.k) + (int64_t)plane * io.bh_stride;
  uint8_t* codes = (is_v ? io.c.v : io.c.k) + (int64_t)plane * io.c.bh_stride + (int64_t)io.first_unit * 4;
  uint8_t* scale = (is_v ? io.c.vs : io.c.ks) + (int64_t)plane * io.c.sc_stride + io.first_unit / 4;
  const int32_t u0 = g * (kNT * kUnits) + threadIdx.x;
  float x[kUnits][8];
#pragma unroll
  for (int j = 0; j < kUnits; ++j) {
    const int32_t u = u0 + j * kNT;
    load8(src + (int64_t)(u < io.units ? u : io.units - 1) * 8, x[j]);
  }
#pragma unroll
  for (int j = 0; j < kUnits; ++j) {
    const int32_t u = u0 + j * kNT;
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t b = __float_as_uint(x[j][i]) & 0x7fffffffu;
      top = b > top ? b : top;
    }
    uint32_t o = (uint32_t)dpp_or_zero<kDppXor1, 0xf>((int32_t)top);
    top = o > top ? o : top;
    o = (uint32_t)dpp_or_zero<kDppXor2, 0xf>((int32_t)top);
    top = o > top ? o : top;
    const uint32_t byte = q4_scale_byte(top);
    const uint32_t w = q4_encode8(x[j], q4_scale(byte));
    if (u < io.units) {  // (whole groups of four lanes)
      *reinterpret_cast<uint32_t*>(codes + (int64_t)u * 4) = w;
      if ((u & 3) == 0) scale[u >> 2] = (uint8_t)byte;
    }
  }
}

struct DequantizeIO {
  void *k, *v;
  int64_t bh_stride;
  Q4View c;
  int32_t units, first_unit, groups;
};

template <class T>
__global__ __launch_bounds__(kNT) void kv_dequantize_q4_kernel(DequantizeIO io) {
  const int32_t g = blockIdx.x % io.groups, rest = blockIdx.x / io.groups;
  const bool is_v = rest & 1;
  const int32_t plane = rest >> 1;
  const uint8_t* codes = (is_v ? io.c.v : io.c.k) + (int64_t)plane * io.c.bh_stride + (int64_t)io.first_unit * 4;
  const uint8_t* scale = (is_v ? io.c.vs : io.c.ks) + (int64_t)plane * io.c.sc_stride + io.first_unit / 4;
  T* dst = static_cast<T*>(is_v ? io.v : io.k) + (int64_t)plane * io.bh_stride;
  const int32_t u0 = g * (kNT * kUnits) + threadIdx.x;
  uint32_t w[kUnits], s[kUnits];
#pragma unroll
  for (int j = 0; j < kUnits; ++j) {
    const int32_t u = u0 + j * kNT, uc = u < io.units ? u : io.units - 1;
    w[j] = *reinterpret_cast<const uint32_t*>(codes + (int64_t)uc * 4);
    s[j] = scale[uc >> 2];
  }
#pragma unroll
  for (int j = 0; j < kUnits; ++j) {
    const int32_t u = u0 + j * kNT;
    if (u >= io.units) continue;
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<u32x4*>(dst + (int64_t)u * 8) = q4_decode8_bf16(w[j], q4_scale(s[j]));
    } else {
      float x[8];
      q4_decode8(w[j], q4_scale(s[j]), x);
      *reinterpret_cast<float4*>(dst + (int64_t)u * 8) = make_float4(x[0], x[1], x[2], x[3]);
      *reinterpret_cast<float4*>(dst + (int64_t)u * 8 + 4) = make_float4(x[4], x[5], x[6], x[7]);
    }
  }
}

int32_t groups_of(int32_t units) { return (int32_t)(((int64_t)units + kNT * kUnits - 1) / (kNT * kUnits)); }

}  // namespace

hipError_t launch_kv_quantize_q4(const KvQuantizeQ4Args& a, hipStream_t stream) {
  QuantizeIO io;
  io.k = a.k;
  io.v = a.v;
  io.bh_stride = a.bh_stride;
  io.c = a.c4;
  io.units = a.n * (a.d / 8);
  io.first_unit = a.t0 * (a.d / 8);
  io.groups = groups_of(io.units);
  const dim3 grid(2 * a.planes * io.groups);
  if (a.bf16) hipLaunchKernelGGL((kv_quantize_q4_kernel<bf16_bits>), grid, dim3(kNT), 0, stream, io);
  else hipLaunchKernelGGL((kv_quantize_q4_kernel<float>), grid, dim3(kNT), 0, stream, io);
  return hipGetLastError();
}

hipError_t launch_kv_dequantize_q4(const KvDequantizeQ4Args& a, hipStream_t stream) {
  DequantizeIO io;
  io.k = a.k;
  io.v = a.v;
  io.bh_stride = a.bh_stride;
  io.c = a.c4;
  io.units = a.n * (a.d / 8);
  io.first_unit = a.t0 * (a.d / 8);
  io.groups = groups_of(io.units);
  const dim3 grid(2 * a.planes * io.groups);
  if (a.bf16) hipLaunchKernelGGL((kv_dequantize_q4_kernel<bf16_bits>), grid, dim3(kNT), 0, stream, io);
  else hipLaunchKernelGGL((kv_dequantize_q4_kernel<float>), grid, dim3(kNT), 0, stream, io);
  return hipGetLastError();
}

}  // namespace sparvar
