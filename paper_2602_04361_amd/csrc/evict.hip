// Eviction: of a plane's tokens the first ones, the last ones and those of largest weight move, in
// order, to a cache of their own.
//
// The largest weights are found by their bits, mapped so that unsigned order is the weights' order.
// Of more than a few tokens a sample tells first between which two weights the threshold lies; of those between,
// a histogram in LDS of the distance to the lower one, its topmost 11 bits, tells those of the
// smallest weight that stays, a second one of the weights that share them the next, until all are
// known, and how many equal to it do (the first ones). Where the sample was wrong the same is done
// between the smallest and the largest weight there is. One launch: every workgroup of a plane finds
// the same threshold and the same places by itself, from the plane's weights, and then copies its own
// run of kept rows, which is what takes the time: it is bound by memory. 2 x 8 heads of 128, 21260 of 42521 tokens,
// bf16: 87 us for 354 MB, a large copy of as much 69, the difference the search of the threshold before it (117 with
// passes over all tokens for every digit, each a histogram of one bin a weight). 460 of 921 tokens of 2 x 12 heads:
// 11 us, all latency. 1024 of 42521 tokens of equal weight 29 us, of different ones 27. Ranks stay in registers up to
// 49152 tokens (12 rows of 4096; 104 registers), past that they are read again in every pass, by each of a plane's workgroups,
// of which there is one for every 4096 kept rows: the search then grows with the square of the length. Half of n tokens
// of 2 x 8 heads of 128 again and again, us (at the copy's rate): 49152 72 (79, partly from the last-level cache), 49153 85,
// 60000 108 (97), 100000 194 (161), 200000 476 (322); one head, 100000 57 (10), 400000 221 (40).
#include "device_common.h"
#include "launch.h"

namespace sparvar {

namespace {

constexpr int kNT = 1024, kNW = kNT / 64;
constexpr int kBins = 2048;
constexpr int kRun = 4096;       // kept rows of a workgroup, at most
constexpr int kSpan = 4 * kNT;   // tokens of a row: four neighbouring ones a thread
constexpr int kTileRows = 16;    // rows that places are counted over at once

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

typedef __attribute__((ext_vector_type(4), aligned(4))) float f32x4_any;  // (at any weight)

// Ranks of four weights. Weights are sums of probabilities: none of a wave's is below zero or NaN but
// for odd inputs, and then their bits need only the topmost set.
__device__ __forceinline__ u32x4 ranks_of(f32x4_any x) {
  u32x4 o;
  bool odd = false;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const uint32_t b = __float_as_uint(x[c]);
    odd |= b > 0x7f800000u;
    o[c] = b | 0x80000000u;
  }
  if (__builtin_amdgcn_ballot_w64(odd)) {
#pragma unroll
    for (int c = 0; c < 4; ++c) o[c] = rank_of(x[c]);
  }
  return o;
}

// Ranks of a thread's tokens (four of each row; those outside [lo, hi) 0): ROWS rows in registers, or
// read again each time.
template <int ROWS>
struct Ranks {
  const float* w;
  int32_t lo, hi;
  u32x4 r[ROWS > 0 ? ROWS : 1];
  __device__ __forceinline__ u32x4 read(int32_t row) const {
    const int32_t at = row * kSpan + 4 * (int32_t)threadIdx.x;
    if (row * kSpan >= lo && (row + 1) * kSpan <= hi) return ranks_of(*reinterpret_cast<const f32x4_any*>(w + at));
    u32x4 o = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int c = 0; c < 4; ++c)
      if (at + c >= lo && at + c < hi) o[c] = rank_of(w[at + c]);
    return o;
  }
  __device__ __forceinline__ void load() {
    if constexpr (ROWS > 0) {
#pragma unroll
      for (int i = 0; i < ROWS; ++i) r[i] = read(i);
    }
  }
  __device__ __forceinline__ u32x4 get(int32_t first, int i) const {
    if constexpr (ROWS > 0) return r[i];
    else return read(first + i);
  }
};

// x that the compiler takes for a new value: comparisons with it are made where they stand, not held
// from a pass before as 48 masks.
__device__ __forceinline__ uint32_t uniform_bits(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }
__device__ __forceinline__ uint32_t fresh(uint32_t x) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+s"(x));
#endif
  return x;
}

// Rows in turn: comparisons or LDS reads of all of them ahead would take a register each.
__device__ __forceinline__ void next_row() { __builtin_amdgcn_sched_barrier(0); }

constexpr int kSample = 128, kLast = 64;
struct EvictLds {
  int32_t list[kRun];
  uint32_t hist[kBins];
  int2 at[kTileRows * kNW];      // of each row and wave: ranks above the threshold, and equal to it (then those before)
  int32_t wt[kNW], above[kNW];
  uint32_t found[3], bound[2];
  uint32_t last[kLast];
  int32_t n_last;
  uint32_t sample[kSample];
  int32_t place[kSample];
};

__device__ __forceinline__ int32_t wave_sum(int32_t x) {
  return __builtin_amdgcn_readlane(wave_incl_scan(x), 63);
}

// The bin, from the top, in which `need` ranks are reached, and how many of it are needed (false:
// there are not so many), and how many it holds. Clears the bins. `over`: ranks above those counted,
// of the wave.
__device__ __forceinline__ bool pick_digit(EvictLds& s, int32_t over, int32_t& need, uint32_t& digit, int32_t& held) {
  const int tid = threadIdx.x, top = kBins - 1 - 2 * tid;
  if ((tid & 63) == 0) s.above[tid >> 6] = over;
  __syncthreads();
  const uint2 h = *reinterpret_cast<const uint2*>(&s.hist[top - 1]);
  *reinterpret_cast<uint2*>(&s.hist[top - 1]) = make_uint2(0u, 0u);
  int32_t all_over = 0;
#pragma unroll
  for (int i = 0; i < kNW; ++i) all_over += s.above[i];
  const int32_t h1 = (int32_t)h.y, h0 = (int32_t)h.x, left = need - all_over;
  int32_t all;
  const int32_t above = block_excl_scan<kNT>(h1 + h0, s.wt, all);
  if (left <= 0 || left > all) return false;  // (the same for all)
  if (above < left && left <= above + h1 + h0) {
    const bool first = left <= above + h1;
    s.found[0] = (uint32_t)(first ? top : top - 1);
    s.found[1] = (uint32_t)(left - above - (first ? 0 : h1));
    s.found[2] = (uint32_t)(first ? h1 : h0);
  }
  __syncthreads();
  digit = s.found[0];
  need = (int32_t)s.found[1];
  held = (int32_t)s.found[2];
  return true;
}

template <int ROWS>
__global__ __launch_bounds__(kNT) void kv_evict_kernel(EvictIO io) {
  __shared__ __attribute__((aligned(16))) EvictLds s;
  const KvEvictArgs& a = io.a;
  const int32_t slice = blockIdx.x % io.slices, plane = blockIdx.x / io.slices;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int32_t* const list = s.list;
  int32_t len = a.n;
  if (a.kv_len) {
    const int32_t l = a.kv_len[plane / a.H_kv];
    len = l < 0 ? 0 : (l < a.n ? l : a.n);
  }
  const float* w = a.w + (int64_t)plane * a.w_bh_stride;
  const int32_t m = len < a.n_keep ? len : a.n_keep;
  const int32_t s0 = slice * io.run, s1 = s0 + io.run < a.n_keep ? s0 + io.run : a.n_keep;  // places of this workgroup
  const int32_t lo = a.n_first, hi = len - a.n_last;  // tokens that compete
  int32_t need = a.n_keep - a.n_first - a.n_last;     // for so many places
  if (len <= a.n_keep || s1 <= lo) {  // (nothing to choose, or not in these places)
    for (int32_t i = s0 + tid; i < s1; i += kNT) list[i - s0] = i;
  } else {
    // The first tokens, then those of the others that stay, then the last tokens.
    for (int32_t i = s0 + tid; i < s1; i += kNT) {
      if (i < lo) list[i - s0] = i;
      else if (i >= lo + need) list[i - s0] = hi + (i - lo - need);
    }
    if (need > 0 && s0 < lo + need) {
      const int32_t many = hi - lo;
      uint32_t from = 1u, upto = 0xffffffffu;  // the threshold lies between
      const bool sampled = many > 4 * kSample;
      uint32_t mine = 0;
      if (sampled && tid < kSample) mine = rank_of(w[lo + (int32_t)((int64_t)tid * many / kSample)]);
      Ranks<ROWS> ranks;
      ranks.w = w, ranks.lo = lo, ranks.hi = hi;
      ranks.load();
      constexpr int R = ROWS > 0 ? ROWS : kTileRows, kUnroll = ROWS > 0 ? ROWS : 4;
      const int32_t tiles = ROWS > 0 ? 1 : (hi + R * kSpan - 1) / (R * kSpan);
      *reinterpret_cast<uint2*>(&s.hist[2 * tid]) = make_uint2(0u, 0u);
      if (sampled) {
        // Descending place of each of a sample, by comparison with all of them; the threshold's is
        // need / many of the way, give or take three and a half standard deviations.
        if (tid < kSample) {
          s.sample[tid] = mine;
          s.place[tid] = 0;
        }
        if (tid < 2) s.bound[tid] = tid == 0 ? from : upto;
        __syncthreads();
        constexpr int kPer = kSample * kSample / kNT;  // comparisons a thread
        const int me = tid % kSample, first = tid / kSample * kPer;
        const uint32_t r = s.sample[me];
        int32_t before = 0;
#pragma unroll
        for (int i = 0; i < kPer; i += 4) {
          const uint4 o = *reinterpret_cast<const uint4*>(&s.sample[first + i]);
          before += (o.x > r || (o.x == r && first + i < me)) ? 1 : 0;
          before += (o.y > r || (o.y == r && first + i + 1 < me)) ? 1 : 0;
          before += (o.z > r || (o.z == r && first + i + 2 < me)) ? 1 : 0;
          before += (o.w > r || (o.w == r && first + i + 3 < me)) ? 1 : 0;
        }
        atomicAdd(&s.place[me], before);
        __syncthreads();
        const float share = (float)need / (float)many, at = share * kSample;
        const float wide = 1.5f + 3.5f * __builtin_sqrtf(at * (1.f - share));
        if (tid < kSample) {
          if (at >= wide && s.place[tid] == (int32_t)(at - wide)) s.bound[1] = mine;
          if (s.place[tid] == (int32_t)(at + wide)) s.bound[0] = mine;
        }
        __syncthreads();
        from = s.bound[0];
        upto = s.bound[1];
      } else {
        __syncthreads();
      }
      // The threshold's distance to the lower end, 11 bits a pass (high: those known, `had` bits left)
      // until few weights share what is known: then by comparison of those.
      uint32_t limit = 0;  // the smallest rank that stays, `need` times
      for (bool again = true; again;) {
        again = false;
        const uint32_t range = upto - from;
        uint32_t high = 0;
        int had = 32 - __builtin_clz(range | 1u);
        int32_t held = 0;
        limit = from;
        for (bool first = true; first || had > 0; first = false) {
          const int next = had > 11 ? had - 11 : 0;
          // ranks that share what is known: `span` from `base` on
          const uint32_t base = fresh(uniform_bits(first ? from : from + (high << had))), top = fresh(uniform_bits(upto));
          const uint32_t rest = top - base, width = (1u << (had & 31)) - 1u, span = first || rest < width ? rest : width;
          int32_t over = 0;
          if (!first && held <= kLast) {
            if (tid == 0) s.n_last = 0;
            __syncthreads();
            for (int32_t t = 0; t < tiles; ++t) {
#pragma unroll kUnroll
              for (int i = 0; i < R; ++i) {
                next_row();
                const u32x4 r = ranks.get(t * R, i);
#pragma unroll
                for (int c = 0; c < 4; ++c)
                  if (r[c] - base <= span) s.last[atomicAdd(&s.n_last, 1)] = r[c];
              }
            }
            __syncthreads();
            if (tid < kLast) {  // (one wave)
              const uint32_t me = lane < held ? s.last[lane] : 0u;
              int32_t above = 0, equal = 0;
              for (int32_t i = 0; i < held; ++i) {
                const uint32_t o = (uint32_t)__builtin_amdgcn_readlane((int)me, i);
                above += o > me ? 1 : 0;
                equal += o == me ? 1 : 0;
              }
              if (lane < held && above < need && need <= above + equal) {  // (those equal to it write the same)
                s.found[0] = me;
                s.found[1] = (uint32_t)(need - above);
                s.found[2] = (uint32_t)equal;
              }
            }
            __syncthreads();
            limit = s.found[0];
            need = (int32_t)s.found[1];
            held = (int32_t)s.found[2];
            break;
          }
          // (those equal to the lower end are counted apart: many equal weights, zeros of keys that got nothing
          // among them, would queue up for one bin)
          int32_t same = 0;
          for (int32_t t = 0; t < tiles; ++t) {
#pragma unroll kUnroll
            for (int i = 0; i < R; ++i) {
              next_row();
              const u32x4 r = ranks.get(t * R, i);
#pragma unroll
              for (int c = 0; c < 4; ++c) {
                over += r[c] > top ? 1 : 0;
                const uint32_t v = r[c] - base;
                same += v == 0u ? 1 : 0;
                if (v - 1u < span) atomicAdd(&s.hist[v >> next], 1u);
              }
            }
          }
          same = wave_sum(same);
          if (lane == 0 && same > 0) atomicAdd(&s.hist[0], (uint32_t)same);
          uint32_t digit;
          if (!pick_digit(s, first ? wave_sum(over) : 0, need, digit, held)) {  // (the first pass of a sample that was wrong)
            from = 1u;
            upto = 0xffffffffu;
            again = true;
            break;
          }
          high = first ? digit : high << (had - next) | digit;
          had = next;
          limit = from + (high << had);
        }
        if (!again && need == held) {  // all that are equal to it stay
          --limit;
          need = 0;
        }
      }
      limit = uniform_bits(limit);
      need = uniform(need);
      // Places of those above it and of the first `need` equal to it
      int32_t gt0 = 0, eq0 = 0;
      for (int32_t t = 0; t < tiles; ++t) {
        __syncthreads();
        int gts = 0, eqs = 0;  // of row `lane`
#pragma unroll kUnroll
        for (int i = 0; i < R; ++i) {
          next_row();
          const u32x4 r = ranks.get(t * R, i);
          const uint32_t lim = fresh(limit);
          int32_t gt = 0, eq = 0;
#pragma unroll
          for (int c = 0; c < 4; ++c) gt += __builtin_popcountll(__builtin_amdgcn_ballot_w64(r[c] > lim));
          if (need > 0) {
#pragma unroll
            for (int c = 0; c < 4; ++c) eq += __builtin_popcountll(__builtin_amdgcn_ballot_w64(r[c] == lim));
          }
          gts = lane == i ? gt : gts;
          eqs = lane == i ? eq : eqs;
        }
        if (lane < R) s.at[lane * kNW + wave] = make_int2(gts, eqs);
        __syncthreads();
        int2 all = make_int2(0, 0);
        if (tid < 64) {  // the first wave adds them up, R * kNW / 64 a lane
          constexpr int kPer = (R * kNW + 63) / 64;
          int2 v[kPer], sum = make_int2(0, 0);
#pragma unroll
          for (int j = 0; j < kPer; ++j) {
            v[j] = lane * kPer + j < R * kNW ? s.at[lane * kPer + j] : make_int2(0, 0);
            sum.x += v[j].x;
            sum.y += v[j].y;
          }
          int2 before = make_int2(wave_incl_scan(sum.x) - sum.x + gt0, wave_incl_scan(sum.y) - sum.y + eq0);
#pragma unroll
          for (int j = 0; j < kPer; ++j) {
            if (lane * kPer + j < R * kNW) s.at[lane * kPer + j] = before;
            before.x += v[j].x;
            before.y += v[j].y;
          }
          if (lane == 63) {
            s.above[0] = before.x;
            s.above[1] = before.y;
          }
        }
        __syncthreads();
        all = make_int2(s.above[0], s.above[1]);
#pragma unroll kUnroll
        for (int i = 0; i < R; ++i) {
          next_row();
          const int2 at = s.at[i * kNW + wave];
          const int32_t g0 = __builtin_amdgcn_readfirstlane(at.x), e0 = __builtin_amdgcn_readfirstlane(at.y);
          const int32_t p0 = lo + g0 + (e0 < need ? e0 : need);
          if (p0 + 256 <= s0 || p0 >= s1) continue;  // (no place of this workgroup's among the wave's)
          next_row();
          const u32x4 r = ranks.get(t * R, i);
          const uint32_t lim = fresh(limit);
          int32_t n = 0;
#pragma unroll
          for (int c = 0; c < 4; ++c) n += r[c] > lim ? 1 : 0;
          if (need > 0) {
#pragma unroll
            for (int c = 0; c < 4; ++c) n += r[c] == lim ? 0x10000 : 0;
          }
          n = wave_incl_scan(n) - n;
          int32_t g = g0 + (n & 0xffff), e = e0 + (n >> 16);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const bool gt = r[c] > lim, eq = r[c] == lim;
            const int32_t p = lo + g + (e < need ? e : need);
            if ((gt || (eq && e < need)) && p >= s0 && p < s1) list[p - s0] = (t * R + i) * kSpan + 4 * tid + c;
            g += gt ? 1 : 0;
            e += eq ? 1 : 0;
          }
        }
        gt0 = all.x;
        eq0 = all.y;
      }
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
  const int32_t rows = (a.n + kSpan - 1) / kSpan;
  if (rows <= 2) hipLaunchKernelGGL((kv_evict_kernel<2>), grid, dim3(kNT), 0, stream, io);
  else if (rows <= 6) hipLaunchKernelGGL((kv_evict_kernel<6>), grid, dim3(kNT), 0, stream, io);
  else if (rows <= 12) hipLaunchKernelGGL((kv_evict_kernel<12>), grid, dim3(kNT), 0, stream, io);
  else hipLaunchKernelGGL((kv_evict_kernel<0>), grid, dim3(kNT), 0, stream, io);
  return hipGetLastError();
}

}  // namespace sparvar
