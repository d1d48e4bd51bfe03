// Attention weight of a cache's keys: w[j] = decay w_old[j] + sum over the queries i of the head
// group of exp(scale q_i k_j - lse_i), lse the log of the softmax denominators that attention gave.
//
// S = Q K^T by MFMA with the queries as rows, so that a lane's column is one key and its registers
// are 16 queries of it: a key's sum stays in a lane (one exchange between the halves at the end),
// and no sum is made by atomics. Half the products of attention, the same exponentials. K is held
// in registers; 4-bit keys become bf16 on their way there, which is exact. Scores, sums and weights
// are held in 32 bits.
//
// A sum over channels may run in any order: a lane's fragments are 16-byte units of its half of a
// row, the same ones of Q (rows in LDS) and K (registers), eight bf16 or four fp32 channels each.
//
// Many rows: bound by the matrix units (55% busy) and the exponentials beside them (vector units 74%). 2 x 16 heads,
// 4096 x 10521, d = 128, bf16 362 to 382 us by card, 0.98 to 0.92 PFLOP/s; with the exponentials of a tile behind
// its products, not under the next tile's, 382 where now 362.
#include "device_common.h"
#include "launch.h"
#include "q4.h"

namespace sparvar {

namespace {

enum class Keys { kBf16, kF32, kQ4 };

struct WeightsIO {
  const char* q;
  const char* k;
  const uint8_t* ks;
  const float* lse;
  const float* w_old;
  float* w;
  const int32_t *kv_len, *old_len;
  int64_t q_bh_stride, k_bh_stride, ks_bh_stride, w_bh_stride;  // bytes (w: elements)
  int32_t n_q, rows, group, H_kv;  // rows = group * n_q: those of a key head
  int32_t n_kv, n_old, slabs;      // workgroups a plane
  int32_t n_items, swizzle;        // workgroups doing work
  int32_t flat;                    // the rows of a group follow one another in memory
  float scale_log2, decay;
};

template <Keys KT>
struct Traits {
  static constexpr int kElem = KT == Keys::kF32 ? 4 : 2;
};

// Byte offset of query row i of a group.
template <int D, int ELEM>
__device__ __forceinline__ int64_t query_at(const WeightsIO& io, int32_t i) {
  if (io.flat) return (int64_t)i * (D * ELEM);
  const int32_t h = i / io.n_q;
  return h * io.q_bh_stride + (int64_t)(i - h * io.n_q) * (D * ELEM);
}

// LSE of row i, the last one's of rows that are not there (these hold its query).
__device__ __forceinline__ float lse_at(const WeightsIO& io, const float* lse, int32_t i) { return lse[i < io.rows ? i : io.rows - 1]; }

// A thread's LSE, of row i, in the exp2 domain to its place in LDS. Rows that had no keys (-inf) add nothing,
// whatever is in their place: +inf makes the weight of every number zero, and `none`, a word 32 rows and a bit a row,
// tells which scores must not count even where they are no numbers. Rows that are not there count for nothing
// beside 2e38 but where the last row's own weight is infinite or NaN and theirs may be; if it had no keys, nor had they.
__device__ __forceinline__ void put_lse(const WeightsIO& io, float l, int32_t i, float* lses, uint32_t* none) {
  lses[threadIdx.x] = l == -INFINITY ? INFINITY : (i < io.rows ? l : 2e38f) * kLog2e;
  const uint64_t b = __builtin_amdgcn_ballot_w64(l == -INFINITY);
  if ((threadIdx.x & 31) == 0) none[threadIdx.x / 32] = (uint32_t)(b >> (threadIdx.x & 32));
}

// Those of a stage.
template <int RS>
struct alignas(16) RowsLds {
  float lse2[RS];
  uint32_t none[RS / 32];
};

// Zeroes the scores of those among four rows: registers 4 g .. of a lane hold rows 8 g + 4 half .. of a tile (none: the
// bits from the lane's first row on). Tiles without such rows cost the branch before it: 64 x 64 364 us (363 without it), 377 with
// one row of a hundred, 390 where all are such.
__device__ __forceinline__ void leave_out(f32x16& st, int g, uint32_t none) {
#pragma unroll
  for (int r = 0; r < 4; ++r) st[4 * g + r] = none & (1u << (8 * g + r)) ? 0.f : st[4 * g + r];
}

// The units of a lane's half of a key, as they lie in memory.
template <Keys KT, int D>
struct RawKey {
  static constexpr int kPieces = KT == Keys::kQ4 ? D / 64 : D * Traits<KT>::kElem / 32;
  u32x4 p[kPieces];
  uint32_t sc;
  __device__ __forceinline__ void load(const char* k, const uint8_t* ks, uint32_t tok, int half) {
    if constexpr (KT == Keys::kQ4) {
#pragma unroll
      for (int i = 0; i < kPieces; ++i) p[i] = ldg16(k + (int64_t)tok * (D / 2) + half * (D / 4) + 16 * i);
      if constexpr (D == 128) sc = *reinterpret_cast<const uint16_t*>(ks + (int64_t)tok * 4 + 2 * half);
      else sc = ks[(int64_t)tok * 2 + half];
    } else {
      constexpr int kHalf = D * Traits<KT>::kElem / 2;
#pragma unroll
      for (int i = 0; i < kPieces; ++i) p[i] = ldg16(k + (int64_t)tok * (2 * kHalf) + half * kHalf + 16 * i);
    }
  }
};

// The same as operands.
template <Keys KT, int D>
struct KeyFrag {
  static constexpr int kUnits = D * Traits<KT>::kElem / 32;  // of a half
  u32x4 u[kUnits];
  __device__ __forceinline__ void take(const RawKey<KT, D>& r) {
    if constexpr (KT == Keys::kQ4) {
#pragma unroll
      for (int i = 0; i < kUnits; ++i) u[i] = q4_decode8_bf16(r.p[i / 4][i & 3], q4_scale((r.sc >> (8 * (i / 4))) & 0xff));
    } else {
#pragma unroll
      for (int i = 0; i < kUnits; ++i) u[i] = r.p[i];
    }
  }
};

template <Keys KT>
__device__ __forceinline__ f32x16 unit_product(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (KT == Keys::kF32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = mfma_f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c);
    return c;
  } else {
    return mfma_bf16(as_bf16x8(a), as_bf16x8(b), c);
  }
}

// LSEs of the 16 rows of a lane's registers, of a tile's 32 in LDS.
struct Lse16 {
  float v[16];
  __device__ __forceinline__ void load(const float* tile, int half) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float4 x = *reinterpret_cast<const float4*>(tile + 8 * j + 4 * half);
      v[4 * j] = x.x, v[4 * j + 1] = x.y, v[4 * j + 2] = x.z, v[4 * j + 3] = x.w;
    }
  }
};

// Keeps the computation of x where it stands.
__device__ __forceinline__ void hold(float& x) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+v"(x));
#endif
}

// Sum of the 16 probabilities of a lane.
__device__ __forceinline__ float tile_sum(const f32x16& st, const Lse16& lse2, float scale_log2) {
  float p[16];
#pragma unroll
  for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[r], scale_log2, -lse2.v[r]));
#pragma unroll
  for (int n = 8; n > 0; n >>= 1)
#pragma unroll
    for (int r = 0; r < n; ++r) p[r] += p[r + n];
  return p[0];
}

// Keys of a plane that are weighed, and those that have a weight from before: of each entry its own number, or `most`.
__device__ __forceinline__ int32_t length_of(const WeightsIO& io, const int32_t* lens, int32_t most, int32_t plane) {
  if (!lens) return most;
  const int32_t len = lens[plane / io.H_kv];
  return len < 0 ? 0 : (len < most ? len : most);
}
__device__ __forceinline__ int32_t length_of(const WeightsIO& io, int32_t plane) { return length_of(io, io.kv_len, io.n_kv, plane); }
__device__ __forceinline__ int32_t old_of(const WeightsIO& io, int32_t plane) { return length_of(io, io.old_len, io.n_old, plane); }

__device__ __forceinline__ float weight_of(const WeightsIO& io, bool had, float old, float sum) {
  return had ? __builtin_fmaf(io.decay, old, sum) : sum;
}
__device__ __forceinline__ void store_weight(const WeightsIO& io, int32_t plane, int32_t key, int32_t n_old, float sum) {
  const int64_t at = (int64_t)plane * io.w_bh_stride + key;
  io.w[at] = weight_of(io, key < n_old, key < n_old ? io.w_old[at] : 0.f, sum);
}

// 16-byte unit u of LDS row r at u ^ this.
template <int U>
__device__ __forceinline__ int row_swizzle(int r) {
  return unit_swizzle(r) & (U - 1);
}

// Many rows: WK waves hold 32 KN keys each, and WR such sets of waves take every WR-th tile of 32
// rows. The rows stream through LDS, RS at a time, two stages.
template <Keys KT, int D, int WK, int WR, int KN>
__global__ __launch_bounds__(WK * WR * 64) __attribute__((amdgpu_waves_per_eu(KN == 1 && KT != Keys::kF32 ? 3 : 2))) void key_weights_kernel(WeightsIO io) {
  // (stages as large as leave the LDS of a CU to as many workgroups as its registers hold)
  constexpr int NT = WK * WR * 64, NW = WK * WR, RS = KN == 2 || WR == 4 ? 128 : 64;
  constexpr int kElem = Traits<KT>::kElem, kRow = D * kElem, U = kRow / 16;
  constexpr int kLoads = RS * U / NT;
  static_assert(RS * U % NT == 0, "a stage must split evenly over the workgroup");
  __shared__ __attribute__((aligned(16))) char stage0[RS * kRow];
  __shared__ __attribute__((aligned(16))) char stage1[RS * kRow];
  __shared__ RowsLds<RS> lses[2];
  __shared__ float sums[WR > 1 ? WR : 1][WK * KN * 32];

  // (the workgroups of a plane on one XCD: its rows are read by all of them)
  const int32_t item = swizzled_item(blockIdx.x, gridDim.x, io.swizzle);
  if (item >= io.n_items) return;
  const int32_t slab = item % io.slabs, plane = item / io.slabs;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, half = lane >> 5, wk = wave % WK, wr = wave / WK;
  const int32_t len = length_of(io, plane);
  const int32_t key0 = slab * (WK * KN * 32);
  if (key0 >= len) return;

  const char* kp = io.k + (int64_t)plane * io.k_bh_stride;
  const uint8_t* ksp = io.ks + (int64_t)plane * io.ks_bh_stride;
  const char* qp = io.q + (int64_t)plane * io.group * io.q_bh_stride;
  const float* lp = io.lse + (int64_t)plane * io.rows;
  const int32_t stages = (io.rows + RS - 1) / RS;
  auto issue = [&](int32_t s, char* to) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int first = (j * NW + wave) * 64, slot = first + lane, r = slot / U;
      const int32_t i = s * RS + r;
      dma16(qp + query_at<D, kElem>(io, i < io.rows ? i : io.rows - 1) + 16 * ((slot % U) ^ row_swizzle<U>(r)), to + first * 16);
    }
  };
  issue(0, stage0);
  if (tid < RS) put_lse(io, lse_at(io, lp, tid), tid, lses[0].lse2, lses[0].none);
  KeyFrag<KT, D> kf[KN];
  {
    RawKey<KT, D> raw[KN];
#pragma unroll
    for (int n = 0; n < KN; ++n) {
      const int32_t key = key0 + (wk * KN + n) * 32 + l32;
      raw[n].load(kp, ksp, (uint32_t)(key < len ? key : len - 1), half);
    }
#pragma unroll
    for (int n = 0; n < KN; ++n) kf[n].take(raw[n]);
  }
  float sum[KN];
#pragma unroll
  for (int n = 0; n < KN; ++n) sum[n] = 0.f;

  // Scores of a tile of rows, and under its products the probabilities of the tile before it, a
  // share after each unit (two waves of a SIMD left to themselves go through their products side by
  // side and then through their exponentials side by side); units are read kAhead early.
  struct Tile {
    f32x16 st[KN];
    Lse16 lse2;
  } even, odd;
  constexpr int kUnits = U / 2, kShare = (16 + kUnits - 1) / kUnits;  // probabilities of a key after a unit
  constexpr int kTiles = RS / 32 / WR, kAhead = 3;
  static_assert(kTiles * 32 * WR == RS, "sets take whole tiles of a stage");
  auto add_up = [&](const Tile& t) {
#pragma unroll
    for (int n = 0; n < KN; ++n) sum[n] += tile_sum(t.st[n], t.lse2, io.scale_log2);
  };
  const int l_row = (wr * 32 + l32) * kRow, sw = row_swizzle<U>(l32);
  auto unit = [&](const char* now, int i) {  // unit i of the wave's tiles of a stage
    return *reinterpret_cast<const u32x4*>(now + l_row + i / kUnits * (WR * 32 * kRow) + 16 * ((half * kUnits + i % kUnits) ^ sw));
  };
  u32x4 ahead[kAhead];
  // (inlined by force: eight copies are more than the compiler inlines, and calls would take the tiles to scratch)
  auto tile = [&](const char* now, const RowsLds<RS>& lse, int t, uint32_t none, Tile& cur, const Tile& before)
                  __attribute__((always_inline)) {
    float part[KN][4];
#pragma unroll
    for (int n = 0; n < KN; ++n) {
      cur.st[n] = zero16();
#pragma unroll
      for (int j = 0; j < 4; ++j) part[n][j] = 0.f;
    }
    cur.lse2.load(lse.lse2 + (t * WR + wr) * 32, half);
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int i = t * kUnits + u;
      const u32x4 a = ahead[i % kAhead];
      if (i + kAhead < kTiles * kUnits) ahead[i % kAhead] = unit(now, i + kAhead);
#pragma unroll
      for (int n = 0; n < KN; ++n) cur.st[n] = unit_product<KT>(a, kf[n].u[u], cur.st[n]);
#pragma unroll
      for (int n = 0; n < KN; ++n)
#pragma unroll
        for (int r = u * kShare; r < (u + 1) * kShare && r < 16; ++r) {
          part[n][r & 3] += __builtin_amdgcn_exp2f(__builtin_fmaf(before.st[n][r], io.scale_log2, -before.lse2.v[r]));
          hold(part[n][r & 3]);
        }
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int n = 0; n < KN; ++n) sum[n] += (part[n][0] + part[n][1]) + (part[n][2] + part[n][3]);
    if (none) {
#pragma unroll
      for (int n = 0; n < KN; ++n)
#pragma unroll
        for (int g = 0; g < 4; ++g) leave_out(cur.st[n], g, none >> (4 * half));
    }
  };
  // no tile before the first: probabilities of zero
#pragma unroll
  for (int n = 0; n < KN; ++n) odd.st[n] = zero16();
#pragma unroll
  for (int r = 0; r < 16; ++r) odd.lse2.v[r] = INFINITY;

  auto step = [&](int32_t s, const char* now, char* then, const RowsLds<RS>& lse, RowsLds<RS>& lse_then, bool first) {
    sync_copies_and_writes();
    float lse_next = 0.f;
    if (s + 1 < stages) {
      issue(s + 1, then);
      if (tid < RS) lse_next = lse_at(io, lp, (s + 1) * RS + tid);
    }
    uint32_t none[kTiles];  // (in scalar registers: held in others, or read at the tiles' ends, 64 x 64 took 382 us for 362)
#pragma unroll
    for (int t = 0; t < kTiles; ++t) none[t] = (uint32_t)uniform((int32_t)lse.none[t * WR + wr]);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) ahead[i] = unit(now, i);
    if constexpr (kTiles == 1) {
      if (first) tile(now, lse, 0, none[0], even, odd);
      else tile(now, lse, 0, none[0], odd, even);
    } else {
#pragma unroll
      for (int t = 0; t < kTiles; t += 2) {
        tile(now, lse, t, none[t], even, odd);
        tile(now, lse, t + 1, none[t + 1], odd, even);
      }
    }
    if (s + 1 < stages && tid < RS) put_lse(io, lse_next, (s + 1) * RS + tid, lse_then.lse2, lse_then.none);
  };
  for (int32_t s = 0; s < stages; s += 2) {
    step(s, stage0, stage1, lses[0], lses[1], true);
    if (s + 1 < stages) step(s + 1, stage1, stage0, lses[1], lses[0], false);
  }
  if (kTiles == 1 && (stages & 1)) add_up(even);
  else add_up(odd);
#pragma unroll
  for (int n = 0; n < KN; ++n) sum[n] = sum_halves(sum[n]);
  const int32_t n_old = old_of(io, plane);
  if constexpr (WR == 1) {
#pragma unroll
    for (int n = 0; n < KN; ++n) {
      const int32_t key = key0 + (wk * KN + n) * 32 + l32;
      if (key < len && half == (n & 1)) store_weight(io, plane, key, n_old, sum[n]);
    }
  } else {
    if (half == 0) {
#pragma unroll
      for (int n = 0; n < KN; ++n) sums[wr][(wk * KN + n) * 32 + l32] = sum[n];
    }
    __syncthreads();
    const int32_t key = key0 + tid;
    if (tid < WK * KN * 32 && key < len) {
      float t = 0.f;
#pragma unroll
      for (int r = 0; r < WR; ++r) t += sums[r][tid];
      store_weight(io, plane, key, n_old, t);
    }
  }
}

// Few rows (up to 128 of a key head; single tokens against a long cache): bound by K's way from
// memory. All rows lie in LDS; every wave walks tiles of 32 keys by itself, the next ones' in flight: one token
// of 4 x 32 heads on 8, up to 42521 keys of 4 bits (84 MB) 20.9 us, a large copy of as much 16.3.
constexpr int kFewWaves = 4;
// (their LDS below 64 KB)
template <Keys KT>
constexpr int kFewRows = KT == Keys::kF32 ? 96 : 128;

template <Keys KT, int D>
__global__ __launch_bounds__(kFewWaves * 64) __attribute__((amdgpu_waves_per_eu(2)))
void key_weights_few_kernel(WeightsIO io, int32_t tiles) {
  constexpr int NT = kFewWaves * 64;
  constexpr int kElem = Traits<KT>::kElem, kRow = D * kElem, U = kRow / 16;
  extern __shared__ __attribute__((aligned(16))) char smem[];  // row tiles, then their LSEs and `none`
  const int32_t slab = blockIdx.x % io.slabs, plane = blockIdx.x / io.slabs;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, half = lane >> 5;
  const int32_t len = length_of(io, plane);
  const int32_t first = slab * tiles, end_tile = (len + 31) / 32, end = first + tiles < end_tile ? first + tiles : end_tile;
  if (first >= end) return;

  const char* kp = io.k + (int64_t)plane * io.k_bh_stride;
  const uint8_t* ksp = io.ks + (int64_t)plane * io.ks_bh_stride;
  const char* qp = io.q + (int64_t)plane * io.group * io.q_bh_stride;
  const float* lp = io.lse + (int64_t)plane * io.rows;
  const int32_t row_tiles = (io.rows + 31) / 32;
  float* lses = reinterpret_cast<float*>(smem + row_tiles * 32 * kRow);
  uint32_t* nones = reinterpret_cast<uint32_t*>(lses + row_tiles * 32);

  constexpr int kDeep = KT == Keys::kQ4 ? 4 : (KT == Keys::kBf16 ? 2 : 1);  // tiles in flight
  RawKey<KT, D> raw[kDeep];
  float old[kDeep];
  const float* wo = io.w_old + (int64_t)plane * io.w_bh_stride;
  const int32_t n_old = old_of(io, plane);
  auto load = [&](int j, int32_t t) {
    const int32_t key = t * 32 + l32;
    raw[j].load(kp, ksp, (uint32_t)(key < len ? key : len - 1), half);
    old[j] = key < n_old ? wo[key] : 0.f;
  };
  int32_t t = first + wave;
#pragma unroll
  for (int j = 0; j < kDeep; ++j)
    if (t + j * kFewWaves < end) load(j, t + j * kFewWaves);
  for (int32_t slot = tid; slot < row_tiles * 32 * U; slot += NT) {
    const int32_t r = slot / U, i = r < io.rows ? r : io.rows - 1;
    const u32x4 v = ldg16(qp + query_at<D, kElem>(io, i) + 16 * (slot % U));
    *reinterpret_cast<u32x4*>(smem + r * kRow + 16 * ((slot % U) ^ row_swizzle<U>(r))) = v;
  }
  if (tid < row_tiles * 32) put_lse(io, lse_at(io, lp, tid), tid, lses, nones);
  __syncthreads();
  const int sw = row_swizzle<U>(l32);
  const uint32_t none_of = nones[lane < row_tiles ? lane : 0];  // (of row tile `lane`)
  while (t < end) {
#pragma unroll
    for (int j = 0; j < kDeep; ++j) {
      if (t >= end) break;
      KeyFrag<KT, D> kf;
      kf.take(raw[j]);
      const float had = old[j];
      if (t + kDeep * kFewWaves < end) load(j, t + kDeep * kFewWaves);
      float sum = 0.f;
      for (int32_t rt = 0; rt < row_tiles; ++rt) {
        const char* row = smem + (rt * 32 + l32) * kRow;
        f32x16 st = zero16();
#pragma unroll
        for (int u = 0; u < U / 2; ++u)
          st = unit_product<KT>(*reinterpret_cast<const u32x4*>(row + 16 * ((half * (U / 2) + u) ^ sw)), kf.u[u], st);
        const uint32_t none = (uint32_t)__builtin_amdgcn_readlane((int)none_of, rt);
        // (eight rows at a time, those that are there)
        const int32_t eights = (io.rows - rt * 32 + 7) / 8;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          if (g >= eights) break;
          if (none >> (8 * g) & 0xff) leave_out(st, g, none >> (4 * half));
          const float4 l = *reinterpret_cast<const float4*>(lses + rt * 32 + 8 * g + 4 * half);
          const float lse2[4] = {l.x, l.y, l.z, l.w};
          float p[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[4 * g + r], io.scale_log2, -lse2[r]));
          sum += (p[0] + p[1]) + (p[2] + p[3]);
        }
      }
      sum = sum_halves(sum);
      const int32_t key = t * 32 + l32;
      if (half == 0 && key < len) io.w[(int64_t)plane * io.w_bh_stride + key] = weight_of(io, key < n_old, had, sum);
      t += kFewWaves;
    }
  }
}

template <Keys KT, int D, int WK, int WR, int KN>
hipError_t launch_many(WeightsIO io, int32_t planes, hipStream_t stream) {
  constexpr int32_t keys = WK * KN * 32;
  io.slabs = (io.n_kv + keys - 1) / keys;
  io.n_items = planes * io.slabs;
  const int32_t grid = io.swizzle ? (io.n_items + 7) / 8 * 8 : io.n_items;
  hipLaunchKernelGGL((key_weights_kernel<KT, D, WK, WR, KN>), dim3(grid), dim3(WK * WR * 64), 0, stream, io);
  return hipGetLastError();
}

// Cost of 32 rows in a form of the kernel of many rows, in us, with m workgroups on the busiest CU: the larger
// of a + b m and c m. Fits to 4096 rows and 10521 keys, 2304 / 6425, 1600 / 4121, 1024 / 2521 (4 to 32 key
// heads) and fewer of either, us at d = 128 by workgroups of 256, 128, 64 and 32 keys (the last two with the rows
// shared out among two and four sets of waves): 2 x 16 heads, 4096 rows 362 / 395 / 456 / 650, 1024 rows 33.6 /
// 31.6 / 38.3 / 54.1; 8 heads, 1024 rows 20.5 / 17.3 / 16.0 / 19.5; one key head of 8, 200 rows of each, 1000
// keys 29.4 / 24.3 / 18.1 / 13.4. (fp32 keys in registers leave no room for 256.)
// d = 64, bf16: 2 x 16 heads, 4096 rows 251 / 260 / 284 / 368; 24 heads, 2102 x 8377 91 / 88 / 95 / 124; 2 x 12 heads,
// 576 x 1497 11.3 / 10.9 / 10.1 / 12.0. fp32, 128 / 64 / 32: the same at d = 64 1491 / 1493 / 1721, 496 / 485 / 558, 42.8 / 35.3 /
// 39.1, 8 heads, 1024 x 2521 41.9 / 41.2 / 37.2; d = 128 2861 / 2925 / 3830, 950 / 941 / 1253, 78.4 / 66.6 / 85.5, 74.6 / 74.6 / 76.8.
// The constants of d = 128 serve fp32 at d = 64 too: of ten sizes the form taken is the best in seven, within 2% in one
// and 11 to 13% above it in two (8 heads, 1024 x 2521, and 4, 1600 x 4121); bf16 at d = 64 2 to 19% above in three, d = 128
// fp32 within 1.4% in all.
struct ManyForm {
  int keys;
  float a, b, c;
};
constexpr ManyForm kManyForms[3][4] = {
    // d = 64, d = 128, fp32
    {{256, 0.f, .325f, .325f}, {128, .05f, .175f, 0.f}, {64, .03f, .1f, 0.f}, {32, .02f, .06f, 0.f}},
    {{256, .1f, .37f, .465f}, {128, .14f, .22f, .277f}, {64, .16f, .075f, .175f}, {32, .07f, .08f, .135f}},
    {{256, INFINITY, 0.f, 0.f}, {128, 0.f, 2.05f, 0.f}, {64, .1f, 1.1f, 0.f}, {32, 0.f, .78f, 0.f}}};

int many_form(bool f32, int d, int32_t planes, int32_t n_kv, int num_cu) {
  int best = 128;
  float least = INFINITY;
  for (const ManyForm& f : kManyForms[f32 ? 2 : d == 128]) {
    const int64_t groups = (int64_t)planes * ((n_kv + f.keys - 1) / f.keys);
    const float m = (float)((groups + num_cu - 1) / num_cu), us = f.a + f.b * m > f.c * m ? f.a + f.b * m : f.c * m;
    if (us < least) {
      least = us;
      best = f.keys;
    }
  }
  return best;
}

template <Keys KT, int D>
hipError_t launch_weights(WeightsIO io, int32_t planes, int num_cu, hipStream_t stream) {
  constexpr int kRow = D * Traits<KT>::kElem;
  if (io.rows <= kFewRows<KT>) {
    const int32_t row_tiles = (io.rows + 31) / 32, all = (io.n_kv + 31) / 32;
    // workgroups of at least a tile a wave, as many as eight a CU
    int64_t tiles = ((int64_t)planes * all + 8 * num_cu - 1) / (8 * num_cu);
    tiles = (tiles + kFewWaves - 1) / kFewWaves * kFewWaves;
    io.slabs = (int32_t)((all + tiles - 1) / tiles);
    const size_t lds = (size_t)row_tiles * (32 * (kRow + 4) + 4);
    hipLaunchKernelGGL((key_weights_few_kernel<KT, D>), dim3(planes * io.slabs), dim3(kFewWaves * 64), lds, stream, io,
                       (int32_t)tiles);
    return hipGetLastError();
  }
  switch (many_form(KT == Keys::kF32, D, planes, io.n_kv, num_cu)) {
    case 256:
      if constexpr (KT != Keys::kF32) return launch_many<KT, D, 4, 1, 2>(io, planes, stream);
      [[fallthrough]];
    case 128: return launch_many<KT, D, 4, 1, 1>(io, planes, stream);
    case 64: return launch_many<KT, D, 2, 2, 1>(io, planes, stream);
    default: return launch_many<KT, D, 1, 4, 1>(io, planes, stream);
  }
}

}  // namespace

int32_t key_weights_form(int32_t B, int32_t H, int32_t H_kv, int32_t n_q, int32_t n_kv, int32_t d, bool f32, int num_cu) {
  const int32_t most = f32 ? kFewRows<Keys::kF32> : kFewRows<Keys::kBf16>;
  return H / H_kv * n_q <= most ? 0 : many_form(f32, d, B * H_kv, n_kv, num_cu);
}

hipError_t launch_key_weights(const KeyWeightsArgs& a, hipStream_t stream) {
  const int32_t elem = a.bf16 ? 2 : 4, group = a.H / a.H_kv;
  WeightsIO io;
  io.q = static_cast<const char*>(a.q);
  io.k = a.k ? static_cast<const char*>(a.k) : reinterpret_cast<const char*>(a.c4.k);
  io.ks = a.k ? nullptr : a.c4.ks;
  io.lse = a.lse;
  io.w_old = a.w_old;
  io.w = a.w;
  io.kv_len = a.kv_len;
  io.old_len = a.old_len;
  io.q_bh_stride = a.q_bh_stride * elem;
  io.k_bh_stride = a.k ? a.k_bh_stride * elem : a.c4.bh_stride;
  io.ks_bh_stride = a.k ? 0 : a.c4.sc_stride;
  io.w_bh_stride = a.w_bh_stride;
  io.n_q = a.n_q;
  io.rows = group * a.n_q;
  io.group = group;
  io.H_kv = a.H_kv;
  io.n_kv = a.n_kv;
  io.n_old = a.n_old;
  io.slabs = io.n_items = 0;
  io.swizzle = a.swizzle;
  io.flat = group == 1 || a.q_bh_stride == (int64_t)a.n_q * a.d;
  io.scale_log2 = a.softmax_scale * kLog2e;
  io.decay = a.decay;
  const int32_t planes = a.B * a.H_kv;
  if (!a.k) return a.d == 128 ? launch_weights<Keys::kQ4, 128>(io, planes, a.num_cu, stream) : launch_weights<Keys::kQ4, 64>(io, planes, a.num_cu, stream);
  if (a.bf16) return a.d == 128 ? launch_weights<Keys::kBf16, 128>(io, planes, a.num_cu, stream) : launch_weights<Keys::kBf16, 64>(io, planes, a.num_cu, stream);
  return a.d == 128 ? launch_weights<Keys::kF32, 128>(io, planes, a.num_cu, stream) : launch_weights<Keys::kF32, 64>(io, planes, a.num_cu, stream);
}

}  // namespace sparvar
