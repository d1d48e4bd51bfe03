// What the attention kernels over caches of codes share (8 and 4 bits): the rows and keys that a
// workgroup takes, dense or from CSR rows, the softmax of a chunk, and how rows are stored or
// handed over in parts.
#pragma once

#include "attn_chunk.h"
#include "attn_sources.h"
#include "launch.h"

namespace sparvar {

// Queries and outputs of a call.
struct RowsIO {
  const bf16_bits* q;
  bf16_bits* o;
  float* lse;
  int64_t q_bh_stride;
  int32_t o_rows;   // rows of an output plane
  int32_t n_items;  // workgroups doing work
  int32_t swizzle;
  float scale_log2;
  float* part_o;    // dense calls in parts: [part, row, D] unnormalised sums, and
  float2* part_ml;  // [part, row] maximum (exp2 domain) and sum
  int32_t rows;     // rows of all output planes
};

// Dense calls: the rows of the query heads that share a key head, head after head, cut
// into slabs; the keys of a batch entry in `parts` runs of whole chunks.
template <int KC>
struct DenseRowsSrc {
  static constexpr bool kSparse = false;
  int32_t n_q, n_kv, H_kv, group, slabs, q_per_wg, parts;
  const int32_t* kv_len;
  template <int NT>
  static constexpr int table_bytes() { return 16; }
  __device__ __forceinline__ int32_t part_of(int32_t item) const { return (item / slabs) % parts; }
  __device__ __forceinline__ QuerySet queries(int32_t item, int wave) const {
    QuerySet s;
    s.bh = item / (slabs * parts);  // plane of keys
    s.qbase = 0;
    s.qnc = n_q;
    s.qstride = 0;
    const int32_t q0 = item % slabs * q_per_wg, rows = group * n_q;
    s.q1 = q0 + q_per_wg < rows ? q0 + q_per_wg : rows;
    s.q0 = q0 + wave * kQPerWave;
    return s;
  }
  __device__ __forceinline__ int32_t kv_plane(const QuerySet& s) const { return s.bh; }
  __device__ __forceinline__ void place(const QuerySet& s, int32_t i, int32_t& plane, int32_t& row) const {
    const int32_t h = i / n_q;
    plane = s.bh * group + h;
    row = i - h * n_q;
  }
  __device__ __forceinline__ DenseCursor<KC> cursor(int32_t item, const QuerySet& s) const {
    int32_t n = n_kv;
    if (kv_len) {
      const int32_t len = kv_len[s.bh / H_kv];
      n = len < 0 ? 0 : (len < n_kv ? len : n_kv);
    }
    const int32_t per = ((n + KC - 1) / KC + parts - 1) / parts * KC, first = part_of(item) * per;
    return DenseCursor<KC>{first, first + per < n ? first + per : n};
  }
};

// Chunks of a CSR row whose blocks are packed: the row's tokens, block after block, cut every 64.
// A block cut at its scale's edge (24 tokens of an 8 x 8 block, say) then takes no more room in a
// chunk than it has tokens, where the block table of the bf16 kernels gives it a chunk: block
// sparse 48 x 36, d = 64, 83% of whose table's slots held a token, 30.5 -> 27.5 us, 32 x 18 with
// 54% 15.7 -> 12.5, 64 x 64 with 98% 120.3 -> 121.4. tok is the token of the lane's slot (the
// last one's past count).
struct PackedChunk {
  uint32_t tok;
  int32_t count;
};

// Token of slot base + step, base the lane's and step the same for all: as one instruction, so that
// no register holds a slot (base is taken again at each load: the compiler would keep every sum).
__device__ __forceinline__ int32_t slot_base(const Chunk&, int32_t slot) { return slot; }
__device__ __forceinline__ uint32_t token_at(const Chunk& c, int32_t base, int32_t step) {
  return (uint32_t)chunk_token(c, chunk_slot(base + step, c.count));
}
__device__ __forceinline__ int32_t slot_base(const PackedChunk&, int32_t slot) {
  int32_t b = slot * 4;
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+v"(b));
#endif
  return b;
}
__device__ __forceinline__ uint32_t token_at(const PackedChunk& c, int32_t base, int32_t step) {
  return (uint32_t)__builtin_amdgcn_ds_bpermute(base + step * 4, (int32_t)c.tok);
}

// Where the blocks of a fill stand: for each that has tokens {first token, first position,
// width of its scale << 8 | its own width, ceil(2^20 / its width)}, and the positions apart.
template <int NT>
struct PackedLds {  // byte offsets
  static constexpr int kInfo = 0;
  static constexpr int kStart = kInfo + NT * 16;
  static constexpr int kWt = kStart + (NT + 1) * 4 + 12;
  static constexpr int kGeo = kWt + 16 * 4;
  static constexpr int kBytes = kGeo + (int)((sizeof(GeoTable) + 15) / 16 * 16);
};

template <int NT>
struct PackedCursor {
  using L = PackedLds<NT>;
  static constexpr int kGroup = NT < 512 ? NT : 511;  // entries of a fill: their count in 9 bits, their tokens in 22
  const int32_t* col;
  int32_t k, pos, end;        // (the queries' scale; blocks are those of scales up to it); entries of the row not yet decoded
  int32_t n, total;           // blocks and tokens of this fill
  int32_t blk, at, stop;      // block of the wave's next position, that position, the end of its part
  char* lds;

  __device__ __forceinline__ bool more() const { return pos < end; }

  // The thread's entry of the next kGroup ones: loaded ahead of what is waited for before fill().
  __device__ __forceinline__ int32_t entry() const {
    const int tid = fresh_tid();
    return tid < kGroup && pos + tid < end ? col[pos + tid] : -1;
  }

  // Decodes the next kGroup entries, a thread each (false: none left). Entries that are no blocks
  // are left out, so that no two blocks share a position.
  __device__ __forceinline__ bool fill(int32_t v) {
    int4* info = reinterpret_cast<int4*>(lds + L::kInfo);
    int32_t* start = reinterpret_cast<int32_t*>(lds + L::kStart);
    const GeoTable& G = *reinterpret_cast<const GeoTable*>(lds + L::kGeo);
    const int tid = fresh_tid();
    total = 0;
    while (pos < end && total == 0) {
      __syncthreads();
      // (a lane holds a scale's bound, so that a search is no chain of reads)
      const int32_t bound = G.NB[(tid & 63) < kMaxScales ? tid & 63 : kMaxScales];
      int l = 1;
      for (int32_t i = 1; i < k; ++i) l += v >= __builtin_amdgcn_readlane(bound, i) ? 1 : 0;
      Tile t{0, 0, 1, 1};
      if (v >= 0 && v < __builtin_amdgcn_readlane(bound, k)) t = block_tile_in(G, l, v);
      const int32_t size = t.nr * t.nc;  // at most 4096
      int32_t sum;
      const int32_t before = block_excl_scan<NT>(size > 0 ? 1 << 22 | size : 0, reinterpret_cast<int32_t*>(lds + L::kWt), sum);
      n = __builtin_amdgcn_readfirstlane((uint32_t)sum >> 22);
      total = __builtin_amdgcn_readfirstlane(sum & 0x3fffff);
      // (last blocks first: the full blocks of late scales then begin on a chunk's first slot, and
      // most chunks hold one; 64 x 64 127 us with the few tokens of the first scales in front)
      if (size > 0) {
        const int32_t i = n - 1 - (before >> 22), first = total - size - (before & 0x3fffff);
        info[i] = make_int4(t.base, first, t.stride << 8 | t.nc, ((1 << 20) + t.nc - 1) / t.nc);
        start[i] = first;
      }
      if (tid == 0) start[n] = total;
      __syncthreads();
      pos += kGroup;
      if (total == 0) v = entry();
    }
    blk = 0;
    at = 0;
    stop = total;
    return total > 0;
  }

  __device__ __forceinline__ int32_t take_part(int s, int ks) {
    const int32_t* start = reinterpret_cast<const int32_t*>(lds + L::kStart);
    const int32_t per = ((total + 63) / 64 + ks - 1) / ks;
    at = s * per * 64;
    stop = at + per * 64 < total ? at + per * 64 : total;
    if (at < total) {
      int32_t upto = 0;
      for (int32_t i = 0; i < n; i += 64) {
        const int32_t j = i + (fresh_tid() & 63);
        upto += __builtin_popcountll(__builtin_amdgcn_ballot_w64(j < n && start[j < n ? j : n] <= at));
      }
      blk = upto - 1;
    }
    return per;
  }

  __device__ __forceinline__ bool next(PackedChunk& c) {
    if (at >= stop) return false;
    const int lane = fresh_tid() & 63;
    const int4* info = reinterpret_cast<const int4*>(lds + L::kInfo);
    const int32_t* start = reinterpret_cast<const int32_t*>(lds + L::kStart);
    c.count = stop - at < 64 ? stop - at : 64;
    // the blocks that begin inside the chunk, at most 63
    const int32_t s = start[blk + 1 + lane < n ? blk + 1 + lane : n];
    const int32_t inside = __builtin_popcountll(__builtin_amdgcn_ballot_w64(blk + 1 + lane < n && s < at + c.count));
    int32_t own = blk;
    for (int32_t i = 0; i < inside; ++i) own += at + lane >= __builtin_amdgcn_readlane(s, i) ? 1 : 0;
    const int4 b = info[own];
    const uint32_t r = (uint32_t)(at + lane - b.y);
    const uint32_t q = __umul24(r, (uint32_t)b.w) >> 20;  // r / width: r < 4096, width <= 64
    c.tok = (uint32_t)b.x + r + __umul24(q, (uint32_t)((b.z >> 8) - (b.z & 0xff)));
    if (c.count < 64) c.tok = lane < c.count ? c.tok : (uint32_t)__builtin_amdgcn_readlane(c.tok, c.count - 1);
    at += 64;
    blk += inside + (__builtin_amdgcn_readlane(s, inside) <= at && blk + 1 + inside < n ? 1 : 0);
    return true;
  }
};

// Restricts a walk to part s of ks; returns the chunks of the longest part.
template <int NT>
__device__ __forceinline__ int32_t take_part(PackedCursor<NT>& c, int s, int ks) { return c.take_part(s, ks); }
template <int KC>
__device__ __forceinline__ int32_t take_part(DenseCursor<KC>& c, int s, int ks) {
  const int32_t chunks = c.n > c.pos ? (c.n - c.pos + KC - 1) / KC : 0, per = (chunks + ks - 1) / ks;
  c.pos += s * per * KC;
  c.n = c.pos + per * KC < c.n ? c.pos + per * KC : c.n;
  return per;
}

struct SparseRowsSrc : SparseSrc<64> {
  int32_t group;
  template <int NT>
  static constexpr int table_bytes() { return PackedLds<NT>::kBytes; }
  template <int NT>
  __device__ __forceinline__ PackedCursor<NT> packed_cursor(int32_t item, char* lds) const {
    const int32_t r = row_of(item);
    PackedCursor<NT> c;
    constexpr int kWords = (int)(sizeof(GeoTable) / 4);
    const int32_t* from = reinterpret_cast<const int32_t*>(&G);  // (the first fill starts with a barrier)
    for (int i = threadIdx.x; i < kWords; i += NT) reinterpret_cast<int32_t*>(lds + PackedLds<NT>::kGeo)[i] = from[i];
    c.col = col_idx;
    c.k = k;
    c.pos = row_ptr[r];
    c.end = row_ptr[r + 1];
    c.lds = lds;
    return c;
  }
  __device__ __forceinline__ int32_t part_of(int32_t) const { return 0; }
  __device__ __forceinline__ int32_t kv_plane(const QuerySet& s) const { return s.bh / group; }
  __device__ __forceinline__ void place(const QuerySet& s, int32_t i, int32_t& plane, int32_t& row) const {
    plane = s.bh;
    row = s.qbase + (i / s.qnc) * s.qstride + i % s.qnc;
  }
};

// Log of the softmax denominator, of a maximum in the exp2 domain and a sum: -inf where there were
// no keys, and NaN where one scored NaN (a sum of NaN is no empty one).
__device__ __forceinline__ float lse_of(float m, float l) {
  return l == 0.f ? -INFINITY : (m + __builtin_log2f(l)) * kLn2;
}

// What a wave found for its rows: the part's unnormalised sums, maximum and sum, or the output.
template <int D>
__device__ __forceinline__ void store_rows(const RowsIO& io, const f32x16 (&acc)[D / 32], float m, float l, bool qvalid, int half,
                                           int32_t plane, int32_t qrow, int32_t part) {
  if (!qvalid) return;
  const int64_t orow = (int64_t)plane * io.o_rows + qrow;
  if (io.part_o) {
    const int64_t prow = (int64_t)part * io.rows + orow;
    float* op = io.part_o + prow * D;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<float4*>(op + 32 * dt + 8 * j + 4 * half) =
            make_float4(acc[dt][4 * j], acc[dt][4 * j + 1], acc[dt][4 * j + 2], acc[dt][4 * j + 3]);
    if (half == 0) io.part_ml[prow] = make_float2(m, l);
    return;
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  bf16_bits* op = io.o + orow * D;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint2 w;
      w.x = pack_bf16x2(acc[dt][4 * j] * inv, acc[dt][4 * j + 1] * inv);
      w.y = pack_bf16x2(acc[dt][4 * j + 2] * inv, acc[dt][4 * j + 3] * inv);
      *reinterpret_cast<uint2*>(op + 32 * dt + 8 * j + 4 * half) = w;
    }
  if (io.lse && half == 0) io.lse[orow] = lse_of(m, l);
}

// V^T fragment of step ks2, channels 32 dt .. of a V tile (rows of D bf16 values).
template <int D, int KC>
struct VOffsets {
  int off[2][D / 32];
  __device__ __forceinline__ void init(int l32, int half, int lane) {
    FragOffsets<D, KC> fo;
    fo.init(l32, half, lane);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {  // (V alone, no K tile before it)
      off[0][i] = fo.v_off[0][i] - KC * D * 2;
      off[1][i] = fo.v_off[1][i] - KC * D * 2;
    }
  }
  __device__ __forceinline__ bf16x8 read(const char* tile, int ks2, int dt) const {
    const i16x4 lo = lds_read_tr(tile + off[0][dt] + ks2 * 16 * D * 2);
    const i16x4 hi = lds_read_tr(tile + off[1][dt] + ks2 * 16 * D * 2);
    u32x4 av;
    av[0] = __builtin_bit_cast(uint32_t, __builtin_shufflevector(lo, lo, 0, 1));
    av[1] = __builtin_bit_cast(uint32_t, __builtin_shufflevector(lo, lo, 2, 3));
    av[2] = __builtin_bit_cast(uint32_t, __builtin_shufflevector(hi, hi, 0, 1));
    av[3] = __builtin_bit_cast(uint32_t, __builtin_shufflevector(hi, hi, 2, 3));
    return as_bf16x8(av);
  }
};

// Softmax of a chunk of scores: masks past count, moves the running maximum when a row's grew
// by more than 2^8 (the sums are rescaled then), and packs the probabilities.
template <int D, int KC>
__device__ __forceinline__ void softmax_chunk(f32x16 (&st)[KC / 32], int32_t count, int half, float scale_log2, float& m_run,
                                              float& l_run, f32x16 (&acc)[D / 32], bf16x8 (&pf)[KC / 16]) {
  if (count < KC) mask_tail<KC>(st, count, half);
  const float mx = row_max<KC>(st, scale_log2);
  if (__builtin_amdgcn_ballot_w64(mx > m_run + 8.f)) {
    const float m_new = fmaxf(m_run, mx);
    const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
    l_run *= alpha;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) acc[i] *= alpha;
    m_run = m_new;
  }
  l_run += exp_pack<KC>(st, scale_log2, m_run, pf);
}

// LDS of one wave, written by some lanes and read by others: its instructions run in
// order, so only the compiler has to keep them so.
__device__ __forceinline__ void wave_fence() {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#endif
}

// The form of a dense call: waves of 32 rows in a workgroup (0: the kernel for few rows, 32 rows a
// workgroup) and sets of them that share its keys, slabs of rows, parts of the keys.
struct DensePlan {
  int waves, sets;
  int32_t slabs, parts, rows;  // rows of a slab
};

// Cost of a form, in us: with m workgroups on the busiest CU, which share it, f0 + f m for starting
// and storing, and a + c m for every 64 keys of a part.
struct DenseForm {
  int waves, sets;
  float f0, f, a, c;
  int32_t rows = 0;  // of a workgroup, where not 32 a wave (few rows: 32)
};
constexpr int kMostParts = 128;

template <int N>
DensePlan plan_dense(const DenseForm (&forms)[N], float token_bytes, int32_t planes, int32_t group, int32_t n_q, int32_t n_kv, int32_t d,
                     int num_cu, bool may_split) {
  const int64_t rows = (int64_t)group * n_q, chunks = ((int64_t)n_kv + 63) / 64;
  const float memory = (float)planes * n_kv * token_bytes * (1.f / 5e6f);
  DensePlan best{0, 1, 1, 1, 32};
  float best_us = INFINITY;
  for (const DenseForm& f : forms) {
    const int64_t per = f.rows ? f.rows : (f.waves ? 32 * f.waves : 32), slabs = (rows + per - 1) / per, items = planes * slabs;
    const int64_t sets = f.sets > 1 ? f.sets : 1;
    auto consider = [&](int64_t parts) {
      if (f.sets > 1 && items > num_cu) return;
      if (parts > 1 && (!may_split || f.sets > 1 || parts > chunks || parts > kMostParts)) return;
      const float m = (float)((items * parts + num_cu - 1) / num_cu), even = (float)(items * parts) / (float)num_cu;
      const float walk = (float)((chunks + parts * sets - 1) / (parts * sets)) * (f.a + f.c * m);
      const float read = memory * (m / even) * (1.f + .25f / m);
      float us = f.f0 + f.f * m + (walk > read ? walk : read);
      if (parts > 1) us += 3.f + .08f * parts + (float)parts * planes * rows * d * (8.f / 6e6f);
      if (us < best_us) {
        best_us = us;
        best = DensePlan{f.waves, f.sets, (int32_t)slabs, (int32_t)parts, (int32_t)per};
      }
    };
    // one part; growing numbers of parts while there is less than one workgroup a CU; whole
    // workgroups a CU
    for (int64_t parts = 1; parts == 1 || items * parts < num_cu; parts += parts < 4 ? 1 : parts / 4) consider(parts);
    for (int64_t m = 1; m <= 8; ++m)
      if (m * num_cu / items > 1) consider(m * num_cu / items);
  }
  return best;
}

inline int32_t padded_grid(const RowsIO& io) { return io.swizzle ? (io.n_items + 7) / 8 * 8 : io.n_items; }

inline int64_t part_floats(int32_t parts, int64_t rows, int32_t d) { return (int64_t)parts * rows * (d + 2); }

// Joins the parts of a call's rows, in order.
hipError_t launch_join_parts(const RowsIO& io, int32_t d, int32_t parts, int num_cu, hipStream_t stream);

}  // namespace sparvar
