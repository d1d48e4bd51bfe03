// Filling a cache: the norms and the rotation of query and key heads as their tokens
// are appended, the 8-bit form of a cache as it is written, and its way back.
//
// All of it is bound by memory: 2 to 4 bytes in and 1 to 4 out for about ten
// operations an element (keys to codes take more, and show it). 2 x 16 heads of 128, bf16:
// append of 4096 tokens to a bf16 cache 44 us, 4.6 TB/s (a large copy reaches 4.8), to an 8-bit
// cache 46 us, 3.6 TB/s; 10521 tokens to codes 48 us, 5.4 TB/s; 2521 tokens back 10 us, 6.1 TB/s
// (the last-level cache holds them). From 32 bits, 4096 tokens to a 32-bit cache 81 us, to an
// 8-bit one 62, 10521 tokens to codes 79, back 75: 4.9 to 5.7 TB/s. A single token is the cost of
// a call, 9 us, 5 of them the kernel. A row of d channels is held by d / 8 lanes of 8 channels,
// so that a row's sum of squares is a few exchanges inside a wave and both channels
// of a rotation pair sit in one lane: lane u of a row has channels [8u, 8u + 8) where
// pairs are neighbours and [4u, 4u + 4) and d/2 + [4u, 4u + 4) where they are halves
// apart; its four pairs are 4u .. 4u + 3 in both.
#include "device_common.h"
#include "launch.h"
#include "q8.h"

namespace sparvar {

namespace {

constexpr int kNT = 256;  // threads of a workgroup that encodes no block

// ------------------------------------------------------------------ eight channels
template <int D, int LAY>
struct Lane8 {
  __device__ __forceinline__ static int a(int u) { return LAY == SPARVAR_ROPE_PAIRS ? 8 * u : 4 * u; }
  __device__ __forceinline__ static int b(int u) { return LAY == SPARVAR_ROPE_PAIRS ? 8 * u + 4 : D / 2 + 4 * u; }
};

template <int D, int LAY>
__device__ __forceinline__ void load8(const bf16_bits* row, int u, float (&x)[8]) {
  u32x4 w;
  if constexpr (LAY == SPARVAR_ROPE_PAIRS) {
    w = ldg16(row + 8 * u);
  } else {
    const uint2 p = *reinterpret_cast<const uint2*>(row + Lane8<D, LAY>::a(u));
    const uint2 q = *reinterpret_cast<const uint2*>(row + Lane8<D, LAY>::b(u));
    w = u32x4{p.x, p.y, q.x, q.y};
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

template <int D, int LAY>
__device__ __forceinline__ void load8(const float* row, int u, float (&x)[8]) {
  const float4 p = *reinterpret_cast<const float4*>(row + Lane8<D, LAY>::a(u));
  const float4 q = *reinterpret_cast<const float4*>(row + Lane8<D, LAY>::b(u));
  x[0] = p.x, x[1] = p.y, x[2] = p.z, x[3] = p.w;
  x[4] = q.x, x[5] = q.y, x[6] = q.z, x[7] = q.w;
}

template <int D, int LAY>
__device__ __forceinline__ void store8(bf16_bits* row, int u, const float (&x)[8]) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
  if constexpr (LAY == SPARVAR_ROPE_PAIRS) {
    *reinterpret_cast<u32x4*>(row + 8 * u) = w;
  } else {
    *reinterpret_cast<uint2*>(row + Lane8<D, LAY>::a(u)) = make_uint2(w[0], w[1]);
    *reinterpret_cast<uint2*>(row + Lane8<D, LAY>::b(u)) = make_uint2(w[2], w[3]);
  }
}

template <int D, int LAY>
__device__ __forceinline__ void store8(float* row, int u, const float (&x)[8]) {
  *reinterpret_cast<float4*>(row + Lane8<D, LAY>::a(u)) = make_float4(x[0], x[1], x[2], x[3]);
  *reinterpret_cast<float4*>(row + Lane8<D, LAY>::b(u)) = make_float4(x[4], x[5], x[6], x[7]);
}

template <int D, int LAY>
__device__ __forceinline__ void load_codes(const uint8_t* row, int u, uint32_t& a, uint32_t& b) {
  a = *reinterpret_cast<const uint32_t*>(row + Lane8<D, LAY>::a(u));
  b = *reinterpret_cast<const uint32_t*>(row + Lane8<D, LAY>::b(u));
}

template <int D, int LAY>
__device__ __forceinline__ void store_codes(uint8_t* row, int u, const float (&x)[8], float inv, bool saturate) {
  uint32_t a, b;
  if (saturate) {
    a = encode4(x, inv);
    b = encode4(x + 4, inv);
  } else {
    a = codes4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
    b = codes4(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv);
  }
  if constexpr (LAY == SPARVAR_ROPE_PAIRS) {
    *reinterpret_cast<uint2*>(row + 8 * u) = make_uint2(a, b);
  } else {
    *reinterpret_cast<uint32_t*>(row + Lane8<D, LAY>::a(u)) = a;
    *reinterpret_cast<uint32_t*>(row + Lane8<D, LAY>::b(u)) = b;
  }
}

// x of another lane by DPP (no trip through LDS): lane ^ 1, lane ^ 2, and mirrored in groups of
// 8 and of 16, which after the steps before stand for lane ^ 4 and lane ^ 8.
constexpr int kDppXor1 = 0xB1, kDppXor2 = 0x4E, kDppMirror8 = 0x141, kDppMirror16 = 0x140;

template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __uint_as_float((uint32_t)dpp_or_zero<CTRL, 0xf>((int32_t)__float_as_uint(x)));
}
template <int CTRL>
__device__ __forceinline__ double dpp(double x) {
  const uint2 w = __builtin_bit_cast(uint2, x);
  const uint2 v = make_uint2((uint32_t)dpp_or_zero<CTRL, 0xf>((int32_t)w.x), (uint32_t)dpp_or_zero<CTRL, 0xf>((int32_t)w.y));
  return __builtin_bit_cast(double, v);
}

// Sum over the LANES (8 or 16) lanes of a row.
template <int LANES, class T>
__device__ __forceinline__ T row_sum(T x) {
  x += dpp<kDppXor1>(x);
  x += dpp<kDppXor2>(x);
  x += dpp<kDppMirror8>(x);
  if constexpr (LANES == 16) x += dpp<kDppMirror16>(x);
  return x;
}

// ------------------------------------------------------------------ norm and rotation
// x * r(x), r of the norm (a NaN in the row makes all of it NaN, so no fmax with eps). Sums of
// squares, roots and quotients in 32 bits.
template <int D>
__device__ __forceinline__ void norm8(float (&x)[8], int32_t norm, float eps) {
  if (norm == SPARVAR_NORM_NONE) return;
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) s = __builtin_fmaf(x[i], x[i], s);
  s = row_sum<D / 8>(s);
  const float l2 = __builtin_sqrtf(s);
  const float r = norm == SPARVAR_NORM_RMS ? 1.f / __builtin_sqrtf(s * (1.f / D) + eps) : 1.f / (l2 < eps ? eps : l2);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] *= r;
}

// w: the lane's eight weights; cs: cos and sin of its four pairs.
template <int LAY>
__device__ __forceinline__ void rotate8(float (&x)[8], const float (&cs)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int a = LAY == SPARVAR_ROPE_PAIRS ? 2 * i : i, b = LAY == SPARVAR_ROPE_PAIRS ? 2 * i + 1 : i + 4;
    const float c = cs[2 * i], s = cs[2 * i + 1];
    const float ya = x[a] * c - x[b] * s, yb = x[a] * s + x[b] * c;
    x[a] = ya;
    x[b] = yb;
  }
}

__device__ __forceinline__ void load_cs(const float* table_row, int u, float (&cs)[8]) {
  const float4 p = *reinterpret_cast<const float4*>(table_row + 8 * u);
  const float4 q = *reinterpret_cast<const float4*>(table_row + 8 * u + 4);
  cs[0] = p.x, cs[1] = p.y, cs[2] = p.z, cs[3] = p.w;
  cs[4] = q.x, cs[5] = q.y, cs[6] = q.z, cs[7] = q.w;
}

template <int D, int LAY>
__device__ __forceinline__ void weigh8(float (&x)[8], const float* w, int u) {
  float t[8];
  load8<D, LAY>(w, u, t);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] *= t[i];
}

// y rounded to odd at 20 bits after the point: cut, with the last bit set where anything was
// cut off. A value so rounded and one more rounding to nearest even with two bits fewer or less
// is the value rounded once.
__device__ __forceinline__ float round_odd(double y) {
  uint2 w = __builtin_bit_cast(uint2, y);
  w.y |= w.x < 1u ? w.x : 1u;
  w.x = 0u;
  return (float)__builtin_bit_cast(double, w);
}

// The whole map of a key on its way to codes, in 64 bits, rounded to odd: codes and exponents
// are then those of the exact map, which 32 bits miss wherever a value lies within their error
// of a tie (about one of a million codes, each off by a step). Append of 4096 tokens, 2 x 16
// heads of 128: 46 us, 43 with the map in 32 bits, 39 without norm, weight and rotation.
template <int D, int LAY>
__device__ __forceinline__ void map_exactly(float (&x)[8], const HeadMap& map, bool weighed, const float (&w)[8],
                                            const float (&cs)[8]) {
  double y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = (double)x[i];
  if (map.norm != SPARVAR_NORM_NONE) {
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) s = __builtin_fma(y[i], y[i], s);
    s = row_sum<D / 8>(s);
    const double eps = (double)map.eps;
    const bool rms = map.norm == SPARVAR_NORM_RMS;
    const double z = rms ? s * (1.0 / D) + eps : s;
    double r;
    if (z > 1e-30 && z < 1e30) {  // 1 / sqrt(z) to 2^-44: the 32-bit one and a Newton step
      const double r0 = (double)__builtin_amdgcn_rsqf((float)z);
      r = r0 * __builtin_fma(-0.5 * z * r0, r0, 1.5);
      if (!rms && r * eps > 1.0) r = 1.0 / eps;
    } else {
      const double root = __builtin_sqrt(z);
      r = 1.0 / (!rms && root < eps ? eps : root);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] *= r;
  }
  if (weighed) {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] *= (double)w[i];
  }
  if (map.cos_sin) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int a = LAY == SPARVAR_ROPE_PAIRS ? 2 * i : i, b = LAY == SPARVAR_ROPE_PAIRS ? 2 * i + 1 : i + 4;
      const double c = (double)cs[2 * i], t = (double)cs[2 * i + 1];
      const double ya = y[a] * c - y[b] * t, yb = y[a] * t + y[b] * c;
      y[a] = ya;
      y[b] = yb;
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = round_odd(y[i]);
}

// ------------------------------------------------------------------ kernels
struct AppendIO {
  const void *q, *k, *v;
  int64_t q_batch, q_token, kv_batch, kv_token;
  void *q_out, *k_cache, *v_cache;
  int64_t cache_bh_stride;
  Q8View c8;
  HeadMap map;
  int32_t H, H_kv, n, t0;
  int32_t n_head_groups, n_token_groups;  // of the row part
  int32_t n_heads;                        // heads of the row part: queries, with a 16-bit cache keys and values too
  int32_t n_blocks;                       // of the encoding part: blocks a plane
  int32_t encode_items;                   // workgroups of the encoding part (they come first)
};

// Rows of the row part: a wave takes 64 / (d / 8) neighbouring tokens of kHeads heads in
// turn, the table's values of its tokens held for all of them.
constexpr int kHeads = 4;

template <class T, int D, int LAY, int NT>
__device__ __forceinline__ void append_rows(const AppendIO& io, int32_t item) {
  constexpr int L = D / 8, kRows = 64 / L;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int u = lane % L;
  const int32_t hg = item % io.n_head_groups, rest = item / io.n_head_groups;
  const int32_t tg = rest % io.n_token_groups, b = rest / io.n_token_groups;
  const int32_t tok = (tg * (NT / 64) + wave) * kRows + lane / L;
  const bool valid = tok < io.n;
  const int32_t i = valid ? tok : io.n - 1;
  const int32_t h0 = hg * kHeads, hn = io.n_heads - h0 < kHeads ? io.n_heads - h0 : kHeads;
  auto source = [&](int32_t h) -> const T* {
    if (h < io.H) return static_cast<const T*>(io.q) + b * io.q_batch + i * io.q_token + (int64_t)h * D;
    h -= io.H;
    const T* p = static_cast<const T*>(h < io.H_kv ? io.k : io.v);
    return p + b * io.kv_batch + i * io.kv_token + (int64_t)(h < io.H_kv ? h : h - io.H_kv) * D;
  };
  float x[kHeads][8], cs[8];
#pragma unroll
  for (int j = 0; j < kHeads; ++j)
    if (j < hn) load8<D, LAY>(source(h0 + j), u, x[j]);
  const bool turn = io.map.cos_sin != nullptr;
  if (turn) load_cs(io.map.cos_sin + (int64_t)(io.t0 + i) * D, u, cs);
#pragma unroll
  for (int j = 0; j < kHeads; ++j) {
    if (j >= hn) break;
    const int32_t h = h0 + j;
    T* dst;
    if (h < io.H + io.H_kv) {
      const bool is_q = h < io.H;
      const float* w = is_q ? io.map.q_weight : io.map.k_weight;
      const int32_t hh = is_q ? h : h - io.H;
      norm8<D>(x[j], io.map.norm, io.map.eps);
      if (w) weigh8<D, LAY>(x[j], w + (int64_t)hh * D, u);
      if (turn) rotate8<LAY>(x[j], cs);
      dst = is_q ? static_cast<T*>(io.q_out) + (((int64_t)b * io.H + h) * io.n + i) * D
                 : static_cast<T*>(io.k_cache) + (int64_t)(b * io.H_kv + hh) * io.cache_bh_stride + (int64_t)(io.t0 + i) * D;
    } else {
      const int32_t hh = h - io.H - io.H_kv;
      dst = static_cast<T*>(io.v_cache) + (int64_t)(b * io.H_kv + hh) * io.cache_bh_stride + (int64_t)(io.t0 + i) * D;
    }
    if (valid) store8<D, LAY>(dst, u, x[j]);
  }
}

// One block of G tokens of a plane, by a workgroup: its rows in registers (PASSES rows a
// lane), mapped, their largest magnitude found, encoded and written. Rows before t0 are
// what the cache holds, rows from t0 + n on are not there.
template <class T, int D, int LAY, int PASSES, int NT, bool MAP>
__device__ __forceinline__ void encode_block(const Q8View& c8, bool is_v, int32_t plane, int32_t j, int32_t t0, int32_t n,
                                             const T* src, int64_t src_token, const HeadMap& map, const float* weight) {
  constexpr int L = D / 8, kRows = NT / L;
  const int u = threadIdx.x % L, r0 = threadIdx.x / L;
  const int32_t G = 1 << c8.lg, first = j << c8.lg, end = t0 + n;
  uint8_t* codes = (is_v ? c8.v : c8.k) + (int64_t)plane * c8.bh_stride;
  uint8_t* scale = (is_v ? c8.vs : c8.ks) + (int64_t)plane * c8.sc_stride + j;
  float x[PASSES][8];
  float top = 0.f;
  float w[8];
  if constexpr (MAP) {
    if (!is_v && weight) load8<D, LAY>(weight, u, w);
  }
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int32_t r = p * kRows + r0, t = first + r;
    if (r < G && t >= t0 && t < end) {
      load8<D, LAY>(src + (int64_t)(t - t0) * src_token, u, x[p]);
    } else if (r < G && t < t0) {
      uint32_t a, b;
      load_codes<D, LAY>(codes + (int64_t)t * D, u, a, b);
      const float s = scale_of_byte(*scale);
      decode4(a, s, x[p]);
      decode4(b, s, x[p] + 4);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[p][i] = 0.f;
    }
  }
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int32_t r = p * kRows + r0, t = first + r;
    if constexpr (MAP) {
      // (whole rows take the branch together, and with them the lanes that exchange)
      if (!is_v && r < G && t >= t0 && t < end) {
        float cs[8];
        if (map.cos_sin) load_cs(map.cos_sin + (int64_t)t * D, u, cs);
        map_exactly<D, LAY>(x[p], map, weight != nullptr, w, cs);
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[p][i]));
  }
  top = fmaxf(top, dpp<kDppXor1>(top));
  top = fmaxf(top, dpp<kDppXor2>(top));
  top = fmaxf(top, dpp<kDppMirror8>(top));
  top = fmaxf(top, dpp<kDppMirror16>(top));
  top = fmaxf(top, __shfl_xor(top, 16));
  top = max_halves(top);
  __shared__ float tops[NT / 64];
  if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) top = fmaxf(top, tops[w]);
  // (the exponent is the workgroup's; below the last one nothing exceeds 448)
  const int32_t e = __builtin_amdgcn_readfirstlane(block_exponent(top));
  const float inv = pow2f(-e);
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int32_t r = p * kRows + r0, t = first + r;
    if (r < G && t < end) store_codes<D, LAY>(codes + (int64_t)t * D, u, x[p], inv, e == kScaleExpMax);
  }
  if (threadIdx.x == 0) *scale = (uint8_t)(e + 127);
}

// PASSES = 0: a 16- or 32-bit cache, row part only. Six waves a SIMD: the map in 64 bits and the
// loads ahead of it would take the registers of four.
template <class T, int D, int LAY, int PASSES, int NT>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(6))) void qkv_append_kernel(AppendIO io) {
  int32_t item = blockIdx.x;
  if constexpr (PASSES > 0) {
    if (item < io.encode_items) {
      const int32_t bi = item % io.n_blocks;
      int32_t rest = item / io.n_blocks;
      const bool is_v = rest & 1;
      rest >>= 1;
      const int32_t h = rest % io.H_kv, b = rest / io.H_kv;
      const T* src = static_cast<const T*>(is_v ? io.v : io.k) + b * io.kv_batch + (int64_t)h * D;
      encode_block<T, D, LAY, PASSES, NT, true>(io.c8, is_v, rest, (io.t0 >> io.c8.lg) + bi, io.t0, io.n, src, io.kv_token,
                                            io.map, io.map.k_weight ? io.map.k_weight + (int64_t)h * D : nullptr);
      return;
    }
    item -= io.encode_items;
  }
  append_rows<T, D, LAY, NT>(io, item);
}

struct QuantizeIO {
  const void *k, *v;
  int64_t bh_stride;
  Q8View c8;
  int32_t n, t0, n_blocks;
};

template <class T, int D, int PASSES, int NT>
__global__ __launch_bounds__(NT) void kv_quantize_kernel(QuantizeIO io) {
  const int32_t bi = blockIdx.x % io.n_blocks, rest = blockIdx.x / io.n_blocks;
  const bool is_v = rest & 1;
  const int32_t plane = rest >> 1;
  const T* src = static_cast<const T*>(is_v ? io.v : io.k) + (int64_t)plane * io.bh_stride;
  encode_block<T, D, SPARVAR_ROPE_PAIRS, PASSES, NT, false>(io.c8, is_v, plane, (io.t0 >> io.c8.lg) + bi, io.t0, io.n, src, D,
                                                        HeadMap{}, nullptr);
}

struct DequantizeIO {
  void *k, *v;
  int64_t bh_stride;
  Q8View c8;
  int32_t n, t0, groups;  // workgroups a plane
};

// A lane turns N neighbouring codes (8 to bf16, 4 to fp32) into 16 bytes, kUnits times.
constexpr int kUnits = 4;

template <class T, int D>
__global__ __launch_bounds__(kNT) void kv_dequantize_kernel(DequantizeIO io) {
  constexpr int N = 16 / (int)sizeof(T);
  const int32_t g = blockIdx.x % io.groups, rest = blockIdx.x / io.groups;
  const bool is_v = rest & 1;
  const int32_t plane = rest >> 1;
  const uint8_t* codes = (is_v ? io.c8.v : io.c8.k) + (int64_t)plane * io.c8.bh_stride + (int64_t)io.t0 * D;
  const uint8_t* scale = (is_v ? io.c8.vs : io.c8.ks) + (int64_t)plane * io.c8.sc_stride;
  T* dst = static_cast<T*>(is_v ? io.v : io.k) + (int64_t)plane * io.bh_stride;
  const int32_t units = io.n * (D / N), u0 = g * (kNT * kUnits) + threadIdx.x;
  uint2 w[kUnits];
  uint32_t s[kUnits];
#pragma unroll
  for (int j = 0; j < kUnits; ++j) {
    const int32_t u = u0 + j * kNT, uc = u < units ? u : units - 1;
    if constexpr (N == 8) w[j] = *reinterpret_cast<const uint2*>(codes + (int64_t)uc * N);
    else w[j].x = *reinterpret_cast<const uint32_t*>(codes + (int64_t)uc * N);
    s[j] = scale[(io.t0 + uc / (D / N)) >> io.c8.lg];
  }
#pragma unroll
  for (int j = 0; j < kUnits; ++j) {
    const int32_t u = u0 + j * kNT;
    if (u >= units) continue;
    const float f = scale_of_byte(s[j]);
    if constexpr (N == 8) {
      uint32_t o[4];
      decode4_bf16(w[j].x, f, o[0], o[1]);
      decode4_bf16(w[j].y, f, o[2], o[3]);
      *reinterpret_cast<u32x4*>(dst + (int64_t)u * N) = u32x4{o[0], o[1], o[2], o[3]};
    } else {
      float x[4];
      decode4(w[j].x, f, x);
      *reinterpret_cast<float4*>(dst + (int64_t)u * N) = make_float4(x[0], x[1], x[2], x[3]);
    }
  }
}

// Threads that encode a block of G rows, d / 8 to a row, two rows each at most: every row more
// costs registers and with them waves that wait for memory side by side (append of 4096 tokens,
// 2 x 16 heads of 128, blocks of 64: two rows a thread 47.4 us, four 50.7).
struct BlockShape {
  int passes, threads;
};
BlockShape block_shape(int32_t lg, int32_t d) {
  const int lanes = (d << lg) / 8;  // 128 .. 2048
  return lanes <= 256 ? BlockShape{1, 256} : BlockShape{2, lanes / 2};
}

template <class T, int D, int LAY>
hipError_t append_with(const AppendIO& io, const BlockShape& b, int32_t grid, hipStream_t stream) {
#define SV_SHAPE(P, NN)                                                                                               \
  if (b.passes == P && b.threads == NN) {                                                                             \
    hipLaunchKernelGGL((qkv_append_kernel<T, D, LAY, P, NN>), dim3(grid), dim3(NN), 0, stream, io);                   \
    return hipGetLastError();                                                                                         \
  }
  SV_SHAPE(0, 256) SV_SHAPE(1, 256) SV_SHAPE(2, 256) SV_SHAPE(2, 512)
  if constexpr (D == 128) {
    SV_SHAPE(2, 1024)
  }
#undef SV_SHAPE
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_qkv_append(const AppendArgs& a, hipStream_t stream) {
  AppendIO io;
  io.q = a.q;
  io.k = a.k;
  io.v = a.v;
  io.q_batch = a.q_batch;
  io.q_token = a.q_token;
  io.kv_batch = a.kv_batch;
  io.kv_token = a.kv_token;
  io.q_out = a.q_out;
  io.k_cache = a.k_cache;
  io.v_cache = a.v_cache;
  io.cache_bh_stride = a.cache_bh_stride;
  io.c8 = a.c8;
  io.map = a.map;
  io.H = a.H;
  io.H_kv = a.H_kv;
  io.n = a.n;
  io.t0 = a.t0;
  io.n_heads = a.q8 ? a.H : a.H + 2 * a.H_kv;
  io.n_head_groups = (io.n_heads + kHeads - 1) / kHeads;
  const BlockShape shape = a.q8 ? block_shape(a.c8.lg, a.d) : BlockShape{0, kNT};
  const int tokens = shape.threads / (a.d / 8);  // of a workgroup of the row part
  io.n_token_groups = (a.n + tokens - 1) / tokens;
  io.n_blocks = a.q8 ? (int32_t)((((int64_t)a.t0 + a.n - 1) >> a.c8.lg) - (a.t0 >> a.c8.lg) + 1) : 0;
  io.encode_items = 2 * a.B * a.H_kv * io.n_blocks;
  const int32_t grid = io.encode_items + a.B * io.n_head_groups * io.n_token_groups;
#define SV_APPEND(TT, BF, DD, LL) \
  if (a.bf16 == BF && a.d == DD && a.map.layout == LL) return append_with<TT, DD, LL>(io, shape, grid, stream);
  SV_APPEND(bf16_bits, true, 64, 0) SV_APPEND(bf16_bits, true, 128, 0) SV_APPEND(bf16_bits, true, 64, 1)
  SV_APPEND(bf16_bits, true, 128, 1) SV_APPEND(float, false, 64, 0) SV_APPEND(float, false, 128, 0)
  SV_APPEND(float, false, 64, 1) SV_APPEND(float, false, 128, 1)
#undef SV_APPEND
  return hipErrorInvalidValue;
}

hipError_t launch_kv_quantize(const KvQuantizeArgs& a, hipStream_t stream) {
  QuantizeIO io;
  io.k = a.k;
  io.v = a.v;
  io.bh_stride = a.bh_stride;
  io.c8 = a.c8;
  io.n = a.n;
  io.t0 = a.t0;
  io.n_blocks = (int32_t)((((int64_t)a.t0 + a.n - 1) >> a.c8.lg) - (a.t0 >> a.c8.lg) + 1);
  const BlockShape shape = block_shape(a.c8.lg, a.d);
  const int32_t grid = 2 * a.planes * io.n_blocks;
#define SV_QUANT(TT, BF, DD, P, NN)                                                                            \
  if (a.bf16 == BF && a.d == DD && shape.passes == P && shape.threads == NN) {                                 \
    hipLaunchKernelGGL((kv_quantize_kernel<TT, DD, P, NN>), dim3(grid), dim3(NN), 0, stream, io);              \
    return hipGetLastError();                                                                                  \
  }
#define SV_QUANT_T(TT, BF)                                                                                     \
  SV_QUANT(TT, BF, 64, 1, 256) SV_QUANT(TT, BF, 64, 2, 256) SV_QUANT(TT, BF, 64, 2, 512)                       \
  SV_QUANT(TT, BF, 128, 1, 256) SV_QUANT(TT, BF, 128, 2, 256) SV_QUANT(TT, BF, 128, 2, 512) SV_QUANT(TT, BF, 128, 2, 1024)
  SV_QUANT_T(bf16_bits, true) SV_QUANT_T(float, false)
#undef SV_QUANT_T
#undef SV_QUANT
  return hipErrorInvalidValue;
}

hipError_t launch_kv_dequantize(const KvDequantizeArgs& a, hipStream_t stream) {
  DequantizeIO io;
  io.k = a.k;
  io.v = a.v;
  io.bh_stride = a.bh_stride;
  io.c8 = a.c8;
  io.n = a.n;
  io.t0 = a.t0;
  const int32_t per = kNT * kUnits * (a.bf16 ? 8 : 4);  // elements of a workgroup
  io.groups = (int32_t)(((int64_t)a.n * a.d + per - 1) / per);
  const int32_t grid = 2 * a.planes * io.groups;
#define SV_DEQUANT(TT, BF, DD)                                                                       \
  if (a.bf16 == BF && a.d == DD) {                                                                   \
    hipLaunchKernelGGL((kv_dequantize_kernel<TT, DD>), dim3(grid), dim3(kNT), 0, stream, io);        \
    return hipGetLastError();                                                                        \
  }
  SV_DEQUANT(bf16_bits, true, 64) SV_DEQUANT(bf16_bits, true, 128) SV_DEQUANT(float, false, 64) SV_DEQUANT(float, false, 128)
#undef SV_DEQUANT
  return hipErrorInvalidValue;
}

}  // namespace sparvar
