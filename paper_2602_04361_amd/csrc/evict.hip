// Eviction: of a plane's tokens the first ones, the last ones and those of largest weight move, in
// order, to a cache of their own.
//
// The largest weights are found by their bits: a weight's 32 bits, mapped so that unsigned order is
// the weights' order, are taken 11, 11 and 10 at a time from the top; a histogram in LDS of those
// that share the digits found so far tells the next digit of the smallest weight that stays, and how
// many equal to it do (the first ones). One launch: every workgroup of a plane finds the same
// threshold and the same places by itself, from the plane's weights, and then copies its own run of
// kept rows, which is what takes the time: it is bound by memory.
#include "device_common.h"
#include "launch.h"

namespace sparvar {

namespace {

constexpr int kNT = 1024, kNW = kNT / 64;
constexpr int kBins = 2048;
constexpr int kRun = 4096;       // kept rows of a workgroup, at most
constexpr int kTileRows = 64;    // rows of kNT weights that places are counted over at once

struct EvictIO {
  KvEvictArgs a;
  int32_t slices, run;  // workgroups a plane, kept rows of each
  int32_t lg;           // 16-byte units of a row, as a power of two
};

// The unsigned order of these is the order of weights; a NaN comes above all, both zeros are one.
// None is 0, which stands for tokens that do not compete.
__device__ __forceinline__ uint32_t rank_of(float w) {
  const uint32_t b = w == 0.f ? 0u : __float_as_uint(w);
  if ((b & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Ranks of a thread's tokens (every kNT-th of the plane, those outside [lo, hi) 0): KPT of them in
// registers, or read again each time.
template <int KPT>
struct Ranks {
  const float* w;
  int32_t lo, hi;
  uint32_t r[KPT > 0 ? KPT : 1];
  __device__ __forceinline__ uint32_t read(int32_t at) const {
    const uint32_t x = rank_of(w[at < hi ? at : hi - 1]);
    return at >= lo && at < hi ? x : 0u;
  }
  __device__ __forceinline__ void load() {
    if constexpr (KPT > 0) {
#pragma unroll
      for (int i = 0; i < KPT; ++i) r[i] = read(i * kNT + (int32_t)threadIdx.x);
    }
  }
  __device__ __forceinline__ uint32_t get(int32_t base, int i) const {
    if constexpr (KPT > 0) return r[i];
    else return read(base + i * kNT + (int32_t)threadIdx.x);
  }
};

template <int KPT>
__global__ __launch_bounds__(kNT) void kv_evict_kernel(EvictIO io) {
  __shared__ uint32_t hist[kBins];
  __shared__ int32_t list[kRun];
  __shared__ int32_t counts[kTileRows * kNW];
  __shared__ int32_t wt[kNW];
  __shared__ uint32_t found[2];
  const KvEvictArgs& a = io.a;
  const int32_t slice = blockIdx.x % io.slices, plane = blockIdx.x / io.slices;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int32_t len = a.n;
  if (a.kv_len) {
    const int32_t l = a.kv_len[plane / a.H_kv];
    len = l < 0 ? 0 : (l < a.n ? l : a.n);
  }
  const float* w = a.w + (int64_t)plane * a.w_bh_stride;
  const int32_t m = len < a.n_keep ? len : a.n_keep;
  const int32_t s0 = slice * io.run, s1 = s0 + io.run < a.n_keep ? s0 + io.run : a.n_keep;  // places of this workgroup
  if (len <= a.n_keep) {
    for (int32_t i = s0 + tid; i < s1; i += kNT) list[i - s0] = i;
  } else {
    const int32_t lo = a.n_first, hi = len - a.n_last;  // tokens that compete
    int32_t need = a.n_keep - a.n_first - a.n_last;     // places that they compete for
    Ranks<KPT> ranks;
    ranks.w = w, ranks.lo = lo, ranks.hi = hi;
    ranks.load();
    constexpr int R = KPT > 0 ? KPT : kTileRows, kUnroll = KPT > 0 ? KPT : 4;
    const int32_t tiles = (len + R * kNT - 1) / (R * kNT);  // (one where the ranks are in registers)
    uint32_t prefix = 0, mask = 0;
    if (need > 0) {
      for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0);
        const uint32_t bins = pass == 2 ? 1024 : 2048;
        hist[tid] = 0;
        hist[tid + kNT] = 0;
        __syncthreads();
        for (int32_t t = 0; t < tiles; ++t) {
          const int32_t base = t * R * kNT;
#pragma unroll kUnroll
          for (int i = 0; i < R; ++i) {
            const uint32_t r = ranks.get(base, i);
            if (r != 0u && (r & mask) == prefix) atomicAdd(&hist[(r >> shift) & (bins - 1)], 1u);
          }
        }
        __syncthreads();
        const int top = kBins - 1 - 2 * tid;
        const int32_t h1 = (int32_t)hist[top], h0 = (int32_t)hist[top - 1];
        int32_t all;
        const int32_t above = block_excl_scan<kNT>(h1 + h0, wt, all);
        if (above < need && need <= above + h1 + h0) {
          const bool first = need <= above + h1;
          found[0] = (uint32_t)(first ? top : top - 1);
          found[1] = (uint32_t)(need - above - (first ? 0 : h1));
        }
        __syncthreads();
        prefix |= found[0] << shift;
        mask |= (bins - 1) << shift;
        need = (int32_t)found[1];
      }
    }
    // Places: the first tokens, then of the others those above the threshold and the first `need`
    // equal to it, then the last tokens.
    const bool some = mask != 0;
    for (int32_t i = tid; i < a.n_first; i += kNT)
      if (i >= s0 && i < s1) list[i - s0] = i;
    for (int32_t i = tid; i < a.n_last; i += kNT) {
      const int32_t p = a.n_keep - a.n_last + i;
      if (p >= s0 && p < s1) list[p - s0] = hi + i;
    }
    int32_t gt0 = 0, eq0 = 0;
    for (int32_t t = 0; some && t < tiles; ++t) {
      const int32_t base = t * R * kNT;
      __syncthreads();
#pragma unroll kUnroll
      for (int i = 0; i < R; ++i) {
        const uint32_t r = ranks.get(base, i);
        const uint64_t gt = __builtin_amdgcn_ballot_w64(r > prefix), eq = __builtin_amdgcn_ballot_w64(r == prefix);
        if (lane == 0) counts[i * kNW + wave] = __builtin_popcountll(gt) | __builtin_popcountll(eq) << 16;
      }
      __syncthreads();
      const int32_t c = tid < R * kNW ? counts[tid] : 0;
      int32_t gts, eqs;
      const int32_t gt_before = block_excl_scan<kNT>(c & 0xffff, wt, gts);
      const int32_t eq_before = block_excl_scan<kNT>(c >> 16, wt, eqs);
      // (a tile holds at most 65536 of each; those before the tile are added below)
      __shared__ int32_t gt_at[kTileRows * kNW], eq_at[kTileRows * kNW];
      if (tid < R * kNW) {
        gt_at[tid] = gt0 + gt_before;
        eq_at[tid] = eq0 + eq_before;
      }
      __syncthreads();
#pragma unroll kUnroll
      for (int i = 0; i < R; ++i) {
        const uint32_t r = ranks.get(base, i);
        const uint64_t gt = __builtin_amdgcn_ballot_w64(r > prefix), eq = __builtin_amdgcn_ballot_w64(r == prefix);
        const uint64_t below = (1ull << lane) - 1;
        const int32_t g = gt_at[i * kNW + wave] + __builtin_popcountll(gt & below);
        const int32_t e = eq_at[i * kNW + wave] + __builtin_popcountll(eq & below);
        if (r > prefix || (r == prefix && e < need)) {
          const int32_t p = a.n_first + g + (e < need ? e : need);
          if (p >= s0 && p < s1) list[p - s0] = base + i * kNT + tid;
        }
      }
      gt0 += gts;
      eq0 += eqs;
    }
  }
  __syncthreads();
  // Kept rows [s0, there) of the plane
  const int32_t there = m < s1 ? m : s1;
  const int64_t out = (int64_t)plane * a.n_keep;
  for (int32_t i = s0 + tid; i < s1; i += kNT) {
    const bool is = i < there;
    const int32_t t = is ? list[i - s0] : -1;
    a.kept[out + i] = t;
    if (is) a.w_out[(int64_t)plane * a.w_out_bh_stride + i] = w[t];
  }
  if (there <= s0) return;
  const int32_t units = (there - s0) << io.lg, in_row = (1 << io.lg) - 1;
  const char* ks = static_cast<const char*>(a.k_src) + (int64_t)plane * a.src_stride;
  const char* vs = static_cast<const char*>(a.v_src) + (int64_t)plane * a.src_stride;
  char* kd = static_cast<char*>(a.k_dst) + (int64_t)plane * a.dst_stride + (int64_t)s0 * a.row;
  char* vd = static_cast<char*>(a.v_dst) + (int64_t)plane * a.dst_stride + (int64_t)s0 * a.row;
  constexpr int kIn = 4;
  for (int32_t u0 = tid; u0 < units; u0 += kNT * kIn) {
    u32x4 k[kIn], v[kIn];
#pragma unroll
    for (int j = 0; j < kIn; ++j) {
      const int32_t u = u0 + j * kNT < units ? u0 + j * kNT : units - 1;
      const int64_t from = (int64_t)list[u >> io.lg] * a.row + 16 * (u & in_row);
      k[j] = ldg16(ks + from);
      v[j] = ldg16(vs + from);
    }
#pragma unroll
    for (int j = 0; j < kIn; ++j) {
      const int32_t u = u0 + j * kNT;
      if (u < units) {
        *reinterpret_cast<u32x4*>(kd + (int64_t)u * 16) = k[j];
        *reinterpret_cast<u32x4*>(vd + (int64_t)u * 16) = v[j];
      }
    }
  }
  if (a.srow) {
    const char* kss = static_cast<const char*>(a.ks_src) + (int64_t)plane * a.ssrc_stride;
    const char* vss = static_cast<const char*>(a.vs_src) + (int64_t)plane * a.ssrc_stride;
    char* ksd = static_cast<char*>(a.ks_dst) + (int64_t)plane * a.sdst_stride + (int64_t)s0 * a.srow;
    char* vsd = static_cast<char*>(a.vs_dst) + (int64_t)plane * a.sdst_stride + (int64_t)s0 * a.srow;
    for (int32_t i = tid; i < there - s0; i += kNT) {
      const int64_t t = list[i];
      if (a.srow == 4) {
        reinterpret_cast<uint32_t*>(ksd)[i] = reinterpret_cast<const uint32_t*>(kss)[t];
        reinterpret_cast<uint32_t*>(vsd)[i] = reinterpret_cast<const uint32_t*>(vss)[t];
      } else {
        reinterpret_cast<uint16_t*>(ksd)[i] = reinterpret_cast<const uint16_t*>(kss)[t];
        reinterpret_cast<uint16_t*>(vsd)[i] = reinterpret_cast<const uint16_t*>(vss)[t];
      }
    }
  }
}

}  // namespace

hipError_t launch_kv_evict(const KvEvictArgs& a, hipStream_t stream) {
  EvictIO io;
  io.a = a;
  const int32_t planes = a.B * a.H_kv;
  io.lg = 0;
  while ((16 << io.lg) < a.row) ++io.lg;
  int32_t slices = (a.num_cu + planes - 1) / planes;
  const int32_t most = (a.n_keep + 63) / 64, least = (int32_t)(((int64_t)a.n_keep + kRun - 1) / kRun);
  slices = slices > most ? most : slices;
  slices = slices < least ? least : slices;
  io.run = (a.n_keep + slices - 1) / slices;
  io.slices = (a.n_keep + io.run - 1) / io.run;
  const dim3 grid((uint32_t)planes * io.slices);
  if (a.n <= 8 * kNT) hipLaunchKernelGGL((kv_evict_kernel<8>), grid, dim3(kNT), 0, stream, io);
  else if (a.n <= 48 * kNT) hipLaunchKernelGGL((kv_evict_kernel<48>), grid, dim3(kNT), 0, stream, io);
  else hipLaunchKernelGGL((kv_evict_kernel<0>), grid, dim3(kNT), 0, stream, io);
  return hipGetLastError();
}

}  // namespace sparvar
