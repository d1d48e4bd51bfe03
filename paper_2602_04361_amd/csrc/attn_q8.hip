// Attention over an 8-bit cache: dense, and block-sparse over CSR rows.
//
// The walk is that of the bf16 kernels (attention.hip): S^T = K Q^T, softmax in the exp2
// domain with a running maximum, O^T += V^T P^T. With K = c 2^e (codes c of e4m3, a
// power-of-two scale a block of tokens) S = sum c 2^e q runs on the codes themselves: the
// 32x32x64 8-bit MFMA takes a scale byte a row, and Q goes in as the sum of two e4m3 values
// (QFragF8), at the same rate as one bf16 product. V becomes bf16 on its way to LDS, once a
// workgroup: c 2^e has 4 significant bits, so the conversion (one instruction for two values,
// the scale its operand) rounds nothing, and O is the bf16 product that a 16-bit cache of the
// same values would have. A lane loads 16 or 32 codes of V of one token, so of one scale.
//
// Large calls are bound by the matrix cores and the softmax's VALU work, which share the clock
// that power allows: 4096 x 10521, 2 x 16 heads, d = 128: 557-611 us from card to card, 1.16-1.27
// PFLOP/s, where a large bf16 matrix product reaches 1.23-1.37; MFMA busy 58% of the cycles, no
// bank conflicts.
// (With K converted to bf16 in LDS as well 633-677 us; with the waves in two groups a phase
// apart, products beside softmax, 575 where this one took 592: not kept.) Few rows against a
// long cache are bound by memory: 4.8 TB/s.
//
// Scores, maxima, sums and O are held in 32 bits. The probabilities are rounded to bf16 for the
// product with V, each off by at most 2^-8 of itself, as in the bf16 kernels (the sum that
// divides them is that of the 32-bit ones): outputs are off by 0.0023 of their size against 64
// bits, 0.0017 of that the rounding of the outputs themselves.
#include "attn_chunk.h"
#include "attn_sources.h"
#include "q8.h"

namespace sparvar {

namespace {

struct Q8IO {
  const bf16_bits* q;
  bf16_bits* o;
  float* lse;
  int64_t q_bh_stride;
  Q8View c;
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
struct DenseQ8Src {
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
  int32_t nb, pos, end;       // ids below nb are blocks; entries of the row not yet decoded
  int32_t n, total;           // blocks and tokens of this fill
  int32_t blk, at, stop;      // block of the wave's next position, that position, the end of its part
  char* lds;

  __device__ __forceinline__ bool more() const { return pos < end; }

  // Decodes the next kGroup entries, a thread each (false: none left). Entries that are no blocks
  // are left out, so that no two blocks share a position.
  __device__ __forceinline__ bool fill() {
    int4* info = reinterpret_cast<int4*>(lds + L::kInfo);
    int32_t* start = reinterpret_cast<int32_t*>(lds + L::kStart);
    const GeoTable& G = *reinterpret_cast<const GeoTable*>(lds + L::kGeo);
    const int tid = fresh_tid();
    total = 0;
    while (pos < end && total == 0) {
      __syncthreads();
      const int32_t v = tid < kGroup && pos + tid < end ? col[pos + tid] : -1;
      Tile t{0, 0, 1, 1};
      if (v >= 0 && v < nb) t = block_tile(G, v);
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

struct SparseQ8Src : SparseSrc<64> {
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
    c.nb = G.NB[k];
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

// Which codes of a wave's 16 rows a lane loads and converts: four lanes take a row, 16 codes
// each (col) and at D = 128 the 16 that lie 64 channels further, so that a token's address and
// scale are found once for both. Eight neighbouring lanes take a row and the one four further,
// whose units lie an odd number of units apart (unit_swizzle): every 16-byte write of theirs
// meets eight different groups of banks.
__device__ __forceinline__ void lane_piece(int lane, int& row, int& col) {
  row = ((lane >> 3) & 3) + ((lane >> 2) & 1) * 4 + (lane >> 5) * 8;
  col = lane & 3;
}

// The two bf16 units of 16 codes times f.
__device__ __forceinline__ void put_piece(char* at0, char* at1, const u32x4& raw, float f) {
  uint32_t w[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) decode4_bf16(raw[i], f, w[2 * i], w[2 * i + 1]);
  *reinterpret_cast<u32x4*>(at0) = u32x4{w[0], w[1], w[2], w[3]};
  *reinterpret_cast<u32x4*>(at1) = u32x4{w[4], w[5], w[6], w[7]};
}

// Log of the softmax denominator, of a maximum in the exp2 domain and a sum: -inf where there were
// no keys, and NaN where one scored NaN (a sum of NaN is no empty one).
__device__ __forceinline__ float lse_of(float m, float l) {
  return l == 0.f ? -INFINITY : (m + __builtin_log2f(l)) * kLn2;
}

// What a wave found for its rows: the part's unnormalised sums, maximum and sum, or the output.
template <int D>
__device__ __forceinline__ void store_rows(const Q8IO& io, const f32x16 (&acc)[D / 32], float m, float l, bool qvalid, int half,
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

// Query fragments for the products with K's codes: the row divided by a power of two (its
// largest magnitude then in (224, 448]) as the sum of two e4m3 values. bf16 has 8 significant
// bits and e4m3 4. What the larger part leaves is at most 16, so the smaller one is stored
// times 2^4, under a scale byte of its own: its last place is 2^-13. The sum is the query itself
// for elements from 2^-6 on, among them all from 2^-13 of the row's largest; below, it is off by
// at most half that place, 2^-14 / 224 < 2^-21 of the largest. Rows of one channel of 100 beside
// normals times 0.1, keys of normals times 4: the split alone, in exact sums, moves the LSE by
// 3e-5 (without the 2^4 by 2e-3). The rate is that of one bf16 product (two e4m3 ones at twice
// its rate), and K needs no conversion. Step t of a half covers channels 64 t + 32 half .. + 32,
// as the K fragments do.
typedef __attribute__((ext_vector_type(8))) int i32x8;

template <int D>
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
        raw[4 * t + i] = ldg16(row + 64 * t + 32 * half + 8 * i);
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

// c += K Q^T over 64 channels: a the codes of 32 keys (scale byte ks of the lane's key). Of the
// queries' scale, byte 0 goes with hi and byte 1 with lo.
template <int D>
__device__ __forceinline__ f32x16 mfma_k(i32x8 a, int32_t ks, const QFragF8<D>& q, int t, f32x16 c) {
#if defined(__HIP_DEVICE_COMPILE__)
  c = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, q.hi[t], c, 0, 0, 0, ks, 0, q.scale);
  c = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, q.lo[t], c, 0, 0, 0, ks, 1, q.scale);
#endif
  return c;
}

__device__ __forceinline__ i32x8 two_units(u32x4 a, u32x4 b) {
  return i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
}

// K codes in LDS: rows of D bytes, 16-byte unit u of row r at u ^ code_swizzle(r): two or four
// rows fill the 256 bytes of the banks, and the same unit of sixteen neighbouring rows lies in
// sixteen different places of them.
template <int D>
__device__ __forceinline__ int code_swizzle(int r) {
  return D == 128 ? (r >> 1) & 7 : (r >> 2) & 3;
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

// QW waves of 32 queries walk the keys in chunks of 64, or (KS > 1) KS such sets, each a part of
// them with LDS of its own, joined through it at the end. While a chunk is computed, the next one's K is
// copied to the other K tile and its V loaded to registers, to be converted into the one V tile
// between two barriers: with one V tile four workgroups of two waves fit a CU's LDS, where two
// tiles leave two (block-sparse 64x64, d = 128: 141 against 171 us, both with K converted).
template <int D, int QW, int KS, class Src>
__global__ __launch_bounds__(QW * KS * 64) __attribute__((amdgpu_waves_per_eu(2))) void attn_q8_kernel(Q8IO io, Src src) {
  constexpr int KC = 64, NT = QW * KS * 64;
  constexpr int kRow = D * 2;                 // bytes of a V row in LDS
  constexpr int kKTile = KC * D, kVTile = KC * kRow;
  constexpr int U8 = D / 16;                  // 16-byte units of a row of codes
  constexpr int kPieces = D / 64;             // 16-code pieces of V a lane takes of a row
  // V rows go to waves 16 at a time, K units 64 at a time; where there are more waves than V
  // rows, the second half of them copies K.
  constexpr bool kHalf = QW * 16 > KC;
  constexpr int kVSteps = kHalf ? 1 : KC / (QW * 16);
  constexpr int kKSteps = KC * U8 / ((kHalf ? QW / 2 : QW) * 64);
  static_assert(kHalf ? QW * 16 == 2 * KC : KC % (QW * 16) == 0, "V rows must split evenly");
  static_assert(KC * U8 % ((kHalf ? QW / 2 : QW) * 64) == 0, "K units must split evenly");
  // (sets hand their sums over through the V tiles and the first K tiles: KS (KS - 1) QW pieces)
  constexpr int kJoin = KS > 1 ? (KS - 1) * QW * (D / 2 / KS) * 256 - kKTile : 0;
  constexpr int kStage = kVTile > kJoin ? kVTile : kJoin;
  __shared__ __attribute__((aligned(16))) char ktile0[KS][kKTile];
  __shared__ __attribute__((aligned(16))) char ktile1[KS][kKTile];
  __shared__ __attribute__((aligned(16))) char vtiles[KS][kStage];
  __shared__ __attribute__((aligned(16))) char tsmem[Src::template table_bytes<NT>()];

  const int32_t item = swizzled_item(blockIdx.x, gridDim.x, io.swizzle);
  if (item >= io.n_items) return;
  const int tid = threadIdx.x;
  const int lane = tid & 63, wave_all = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, half = lane >> 5;
  const int split = wave_all / QW, wave = wave_all % QW;

  const QuerySet qs = src.queries(item, wave);
  QFragF8<D> qf;
  {
    int32_t plane, qrow;
    src.place(qs, qs.q0 + l32 < qs.q1 ? qs.q0 + l32 : 0, plane, qrow);
    qf.load(io.q + (int64_t)plane * io.q_bh_stride + (int64_t)qrow * D, half);
  }
  const int32_t kvp = src.kv_plane(qs);
  const uint8_t* kp = io.c.k + (int64_t)kvp * io.c.bh_stride;
  const uint8_t* vp = io.c.v + (int64_t)kvp * io.c.bh_stride;
  const uint8_t* ksp = io.c.ks + (int64_t)kvp * io.c.sc_stride;
  const uint8_t* vsp = io.c.vs + (int64_t)kvp * io.c.sc_stride;

  f32x16 acc[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) acc[i] = zero16();
  float m_run = kNoMax, l_run = 0.f;

  // K fragments: unit 4 t + 2 half + x of row l32 (rows 32 apart share their swizzle)
  int k_off[D / 64][2];
#pragma unroll
  for (int t = 0; t < D / 64; ++t)
#pragma unroll
    for (int x = 0; x < 2; ++x) k_off[t][x] = l32 * D + 16 * ((4 * t + 2 * half + x) ^ code_swizzle<D>(l32));
  VOffsets<D, KC> vo;
  vo.init(l32, half, lane);

  // V: a lane's pieces of row vrow, and of rows QW * 16 further (a multiple of 16, so LDS
  // offsets differ by a constant)
  char* const vtile = vtiles[split];
  int vrow, vcol;
  lane_piece(lane, vrow, vcol);
  vrow += wave * 16;
  const bool does_v = !kHalf || wave < QW / 2, does_k = !kHalf || wave >= QW / 2;  // wave-uniform
  int v_lds[kPieces][2];
#pragma unroll
  for (int p = 0; p < kPieces; ++p)
#pragma unroll
    for (int x = 0; x < 2; ++x)
      v_lds[p][x] = vrow * kRow + 16 * ((2 * (vcol + 4 * p) + x) ^ (unit_swizzle(vrow) & (D / 8 - 1)));
  // K: a direct copy of the wave covers 64 units in a row; a lane fetches the unit that the
  // swizzle puts at its place
  const int k_first = (kHalf ? wave - QW / 2 : wave) * kKSteps * 64;
  const int k_row = (k_first + lane) / U8, k_unit = (k_first + lane) % U8;

  u32x4 raw[kVSteps][kPieces];
  uint32_t raw_s[kVSteps], k_scale[KC / 32], k_scale_next[KC / 32];
  auto load = [&](const auto& c, char* kdst) {
    if (does_k) {
      const int32_t base = slot_base(c, k_row);
#pragma unroll
      for (int j = 0; j < kKSteps; ++j) {
        const int r = k_row + j * (64 / U8);
        const uint32_t tok = token_at(c, base, j * (64 / U8));
        dma16(kp + (tok * D + 16 * (k_unit ^ code_swizzle<D>(r))), kdst + (k_first + j * 64) * 16);
      }
    }
    if (does_v) {
      const int32_t base = slot_base(c, vrow);
#pragma unroll
      for (int j = 0; j < kVSteps; ++j) {
        const uint32_t tok = token_at(c, base, j * QW * 16);
#pragma unroll
        for (int p = 0; p < kPieces; ++p)
          raw[j][p] = *reinterpret_cast<const u32x4*>(vp + (tok * D + 16 * vcol + 64 * p));
        raw_s[j] = vsp[tok >> io.c.lg];
      }
    }
    if constexpr (Src::kSparse) {  // (the tokens of slots l32 and 32 + l32)
      const auto t = __builtin_amdgcn_permlane32_swap(c.tok, c.tok, false, false);
      k_scale_next[0] = ksp[(uint32_t)t[0] >> io.c.lg];
      k_scale_next[1] = ksp[(uint32_t)t[1] >> io.c.lg];
    } else {
#pragma unroll
      for (int kt = 0; kt < KC / 32; ++kt) k_scale_next[kt] = ksp[token_at(c, l32, 32 * kt) >> io.c.lg];
    }
  };
  // The chunk loaded last becomes the one to be computed: V to LDS, K's copies arrived.
  auto take = [&]() {
    if (does_v) {
#pragma unroll
      for (int j = 0; j < kVSteps; ++j)
#pragma unroll
        for (int p = 0; p < kPieces; ++p)
          put_piece(vtile + v_lds[p][0] + j * (QW * 16 * kRow), vtile + v_lds[p][1] + j * (QW * 16 * kRow), raw[j][p],
                    scale_of_byte(raw_s[j]));
    }
#pragma unroll
    for (int kt = 0; kt < KC / 32; ++kt) k_scale[kt] = k_scale_next[kt];
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
  };

  // One chunk, K in kt_, V in vtile; `next` issues the loads of the next one. The order of the
  // LDS reads is pinned: K first, V under the products of S.
  auto compute = [&](const char* kt_, int32_t count, auto next) {
    f32x16 st[KC / 32];
    i32x8 kf[KC / 32][D / 64];
    bf16x8 vf[KC / 16][D / 32], pf[KC / 16];
#pragma unroll
    for (int kt = 0; kt < KC / 32; ++kt)
#pragma unroll
      for (int t = 0; t < D / 64; ++t)
        kf[kt][t] = two_units(*reinterpret_cast<const u32x4*>(kt_ + k_off[t][0] + kt * 32 * D),
                              *reinterpret_cast<const u32x4*>(kt_ + k_off[t][1] + kt * 32 * D));
    __builtin_amdgcn_sched_barrier(0);
    next();
    __builtin_amdgcn_sched_barrier(0);
    constexpr int kProducts = KC / 32 * (D / 64), kV = KC / 16 * (D / 32);  // V fragments to read under them
#pragma unroll
    for (int kt = 0; kt < KC / 32; ++kt) st[kt] = zero16();
#pragma unroll
    for (int i = 0; i < kProducts; ++i) {
      const int kt = i / (D / 64), t = i % (D / 64);
      st[kt] = mfma_k<D>(kf[kt][t], (int32_t)k_scale[kt], qf, t, st[kt]);
#pragma unroll
      for (int f = kV * i / kProducts; f < kV * (i + 1) / kProducts; ++f)
        vf[f / (D / 32)][f % (D / 32)] = vo.read(vtile, f / (D / 32), f % (D / 32));
      __builtin_amdgcn_sched_barrier(0);
    }
    softmax_chunk<D, KC>(st, count, half, io.scale_log2, m_run, l_run, acc, pf);
#pragma unroll
    for (int ks = 0; ks < KC / 16; ++ks)
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) acc[dt] = mfma_bf16(vf[ks][dt], pf[ks], acc[dt]);
  };

  auto cur = [&]() {
    if constexpr (Src::kSparse) return src.template packed_cursor<NT>(item, tsmem);
    else return src.cursor(item, qs);
  }();
  // One pass over what the cursor holds, or over the set's part of it (a block table is filled
  // again between passes, with a barrier, so the tiles are free when a pass starts). Every
  // wave takes the steps of the longest part, and the barriers in them.
  auto walk = [&]() {
    int32_t steps = 0;
    if constexpr (KS > 1) steps = take_part(cur, split, KS);
    std::conditional_t<Src::kSparse, PackedChunk, Chunk> c0;
    bool have = cur.next(c0);
    if (KS == 1 && !have) return;
    if (have) load(c0, ktile0[split]);
    auto step = [&](const char* now, char* then, bool first) -> bool {
      if (!first) __syncthreads();  // V and the other K tile have been read
      if (have) take();
      __syncthreads();
      if (have) {
        const int32_t count = c0.count;
        compute(now, count, [&]() {
          have = cur.next(c0);
          if (have) load(c0, then);
        });
      }
      return KS > 1 ? --steps > 0 : have;
    };
    if (KS > 1 && steps <= 0) return;
    for (bool first = true;; first = false) {
      if (!step(ktile0[split], ktile1[split], first)) break;
      if (!step(ktile1[split], ktile0[split], false)) break;
    }
  };
  if constexpr (Src::kSparse) {
    while (cur.fill()) {
      walk();
      if (!cur.more()) break;
    }
  } else {
    walk();
  }

  // (the rows' places are found again, not held through the walk)
  const int32_t qslot = qs.q0 + (fresh_tid() & 31);
  const bool qvalid = qslot < qs.q1;
  int32_t plane, qrow;
  src.place(qs, qvalid ? qslot : 0, plane, qrow);
  if constexpr (KS > 1) {
    __shared__ float ml[KS][QW * kQPerWave][2];
    float m_g, l_g, out[D / 2 / KS];
    merge_key_splits<D, QW, KS, KS * kStage, KS * kKTile>(acc, m_run, l_run, split, wave, lane, vtiles[0], ktile0[0], ml, m_g,
                                                          l_g, out);
    if (!qvalid) return;
    const float inv = l_g > 0.f ? 1.f / l_g : 0.f;
    const int64_t orow = (int64_t)plane * io.o_rows + qrow;
#pragma unroll
    for (int i = 0; i < D / 8 / KS; ++i) {
      uint2 w;
      w.x = pack_bf16x2(out[4 * i] * inv, out[4 * i + 1] * inv);
      w.y = pack_bf16x2(out[4 * i + 2] * inv, out[4 * i + 3] * inv);
      *reinterpret_cast<uint2*>(io.o + orow * D + channel_of(split * (D / 8 / KS) + i, half)) = w;
    }
    if (io.lse && split == 0 && half == 0) io.lse[orow] = lse_of(m_g, l_g);
    return;
  }
  const float l_tot = sum_halves(l_run);
  store_rows<D>(io, acc, m_run, l_tot, qvalid, half, plane, qrow, src.part_of(item));
}

// Few rows (single tokens against a long cache, a token a query head; early scales): bound by
// memory or latency, so every wave walks chunks of 32 keys by itself, without barriers, its next
// chunk's codes in flight. K goes from registers to the products (converted: splitting the
// queries in two would take longer than a short walk saves, 64 x 121 keys 5.8 against 7.4 us):
// a lane holds half of a key's channels, and as a sum over channels may run in any order, step
// s takes channels 8 s .. of each half. V goes through a piece of LDS of the wave's own, for the
// transposing read. The four waves of a workgroup take every fourth chunk of a part and join
// at the end. One token of 4 x 32 heads, up to 42521 keys of 8 heads: 58.5 us, 4.8 TB/s (a large
// copy reaches 4.8); by the 64-key kernel with parts 91 us.
constexpr int kRowWaves = 4;

// LDS of one wave, written by some lanes and read by others: its instructions run in
// order, so only the compiler has to keep them so.
__device__ __forceinline__ void wave_fence() {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#endif
}

template <int D>
__global__ __launch_bounds__(kRowWaves * 64) __attribute__((amdgpu_waves_per_eu(2)))
void attn_q8_rows_kernel(Q8IO io, DenseQ8Src<32> src) {
  constexpr int KC = 32, kRow = D * 2;
  constexpr int kK = D / 32;             // 16-byte pieces of a lane's half of a key
  constexpr int kPieces = D / 64;        // 16-code pieces of V a lane takes of a row
  constexpr int kTile = KC * kRow;
  __shared__ __attribute__((aligned(16))) char tiles[kRowWaves][kTile];
  __shared__ float2 ml[kRowWaves][32];

  const int32_t item = swizzled_item(blockIdx.x, gridDim.x, io.swizzle);
  if (item >= io.n_items) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l32 = lane & 31, half = lane >> 5;

  const QuerySet qs = src.queries(item, 0);
  const bool qvalid = qs.q0 + l32 < qs.q1;
  int32_t plane, qrow;
  src.place(qs, qvalid ? qs.q0 + l32 : qs.q0, plane, qrow);
  const bf16_bits* q = io.q + (int64_t)plane * io.q_bh_stride + (int64_t)qrow * D + half * (D / 2);
  bf16x8 qf[D / 16];
#pragma unroll
  for (int s = 0; s < D / 16; ++s) qf[s] = as_bf16x8(ldg16(q + 8 * s));

  const uint8_t* kp = io.c.k + (int64_t)qs.bh * io.c.bh_stride;
  const uint8_t* vp = io.c.v + (int64_t)qs.bh * io.c.bh_stride;
  const uint8_t* ks = io.c.ks + (int64_t)qs.bh * io.c.sc_stride;
  const uint8_t* vs = io.c.vs + (int64_t)qs.bh * io.c.sc_stride;

  f32x16 acc[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) acc[i] = zero16();
  float m_run = kNoMax, l_run = 0.f;

  // V: a lane's pieces of rows vrow and vrow + 16
  char* tile = tiles[wave];
  VOffsets<D, KC> vo;
  vo.init(l32, half, lane);
  int vrow, vcol;
  lane_piece(lane, vrow, vcol);
  const int sw = unit_swizzle(vrow) & (D / 8 - 1);

  u32x4 kr[kK], vr[2][kPieces];
  uint32_t ksc, vsc[2];
  const DenseCursor<KC> cur = src.cursor(item, qs);
  auto load = [&](int32_t pos) {
    const int32_t last = cur.n - 1;
    const int32_t kt = pos + l32 < last ? pos + l32 : last;
#pragma unroll
    for (int i = 0; i < kK; ++i)
      kr[i] = *reinterpret_cast<const u32x4*>(kp + ((uint32_t)kt * D + half * (D / 2) + 16 * i));
    ksc = ks[(uint32_t)kt >> io.c.lg];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int32_t r = pos + vrow + 16 * j, vt = r < last ? r : last;
#pragma unroll
      for (int p = 0; p < kPieces; ++p)
        vr[j][p] = *reinterpret_cast<const u32x4*>(vp + ((uint32_t)vt * D + 16 * vcol + 64 * p));
      vsc[j] = vs[(uint32_t)vt >> io.c.lg];
    }
  };
  int32_t pos = cur.pos + wave * KC;
  if (pos < cur.n) load(pos);
  while (pos < cur.n) {
    // V to LDS, K to the products
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int p = 0; p < kPieces; ++p) {
        char* at = tile + (vrow + 16 * j) * kRow;
        put_piece(at + 16 * ((2 * (vcol + 4 * p)) ^ sw), at + 16 * ((2 * (vcol + 4 * p) + 1) ^ sw), vr[j][p],
                  scale_of_byte(vsc[j]));
      }
    wave_fence();
    f32x16 st[1] = {zero16()};
    const float fk = scale_of_byte(ksc);
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      uint32_t w0, w1, w2, w3;
      decode4_bf16(kr[s / 2][2 * (s & 1)], fk, w0, w1);
      decode4_bf16(kr[s / 2][2 * (s & 1) + 1], fk, w2, w3);
      st[0] = mfma_bf16(as_bf16x8(u32x4{w0, w1, w2, w3}), qf[s], st[0]);
    }
    const int32_t count = cur.n - pos;
    pos += kRowWaves * KC;
    if (pos < cur.n) load(pos);
    bf16x8 pf[KC / 16];
    softmax_chunk<D, KC>(st, count, half, io.scale_log2, m_run, l_run, acc, pf);
#pragma unroll
    for (int s2 = 0; s2 < KC / 16; ++s2)
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) acc[dt] = mfma_bf16(vo.read(tile, s2, dt), pf[s2], acc[dt]);
    wave_fence();
  }

  // Join the waves: the row's maximum and sum, then each wave's registers 32 at a time
  // through the tiles; wave w finishes eight of each 32, in wave order.
  const float l_own = sum_halves(l_run);
  if (half == 0) ml[wave][l32] = make_float2(m_run, l_own);
  __syncthreads();
  float m_g = kNoMax, l_g = 0.f;
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) m_g = fmaxf(m_g, ml[w][l32].x);
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) l_g += ml[w][l32].y * __builtin_amdgcn_exp2f(ml[w][l32].x - m_g);
  const float own = __builtin_amdgcn_exp2f(m_run - m_g);
  const float inv = io.part_o ? 1.f : (l_g > 0.f ? 1.f / l_g : 0.f);
  const int64_t orow = (int64_t)plane * io.o_rows + qrow;
  const int64_t prow = (int64_t)src.part_of(item) * io.rows + orow;
  constexpr int kPass = kTile / 256;  // registers of a lane that a tile holds: 32 (D = 128) or 16
#pragma unroll
  for (int p = 0; p < D / 2 / kPass; ++p) {
    if (p > 0) __syncthreads();
    float* to = reinterpret_cast<float*>(tile) + lane;
#pragma unroll
    for (int i = 0; i < kPass; ++i) to[i * 64] = acc[(p * kPass + i) / 16][(p * kPass + i) % 16] * own;
    __syncthreads();
    if (!qvalid) continue;
#pragma unroll
    for (int g = 0; g < kPass / 16; ++g) {  // four registers are four neighbouring channels
      const int i = (wave * (kPass / 16) + g) * 4;
      float r[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kRowWaves; ++w)
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] += reinterpret_cast<const float*>(tiles[w])[(i + e) * 64 + lane];
      const int reg = p * kPass + i, ch = 32 * (reg >> 4) + 8 * ((reg >> 2) & 3) + 4 * half;
      if (io.part_o) {
        *reinterpret_cast<float4*>(io.part_o + prow * D + ch) = make_float4(r[0], r[1], r[2], r[3]);
      } else {
        uint2 w;
        w.x = pack_bf16x2(r[0] * inv, r[1] * inv);
        w.y = pack_bf16x2(r[2] * inv, r[3] * inv);
        *reinterpret_cast<uint2*>(io.o + orow * D + ch) = w;
      }
    }
  }
  if (qvalid && wave == 0 && half == 0) {
    if (io.part_o) io.part_ml[prow] = make_float2(m_g, l_g);
    else if (io.lse) io.lse[orow] = lse_of(m_g, l_g);
  }
}

// Joins the parts of a row: D / 4 channel groups times `side` threads that take every side-th
// part, added in order through LDS; a workgroup of 256 threads takes as many rows as that leaves.
// A part without keys has no sum and its values do not count (a NaN sum is one: its row is NaN in
// every form). Few parts of many rows go a thread a channel group (side = 1, memory bound); else
// a row's parts go side by side (ALL: latency, the token case's 16 parts of 128 rows are 1 MB, 5
// us with the launch). A whole call of 32768 rows of 64 channels in two parts takes 40 us that
// way, 60 with a workgroup a row; 9040 rows in three 28.6 and 34.
template <int D, bool ALL>
__global__ __launch_bounds__(256) void join_parts_kernel(Q8IO io, int32_t parts) {
  constexpr int C = D / 4, P = 256 / C, side = ALL ? P : 1;
  __shared__ float4 sums[ALL ? P : 1][C];
  __shared__ float ls[P];
  const int c = threadIdx.x % C, g = threadIdx.x / C;
  const int32_t row = ALL ? (int32_t)blockIdx.x : (int32_t)blockIdx.x * P + g;
  if (!ALL && row >= io.rows) return;
  float m = kNoMax;
  if constexpr (ALL) {
    for (int p = threadIdx.x & 63; p < parts; p += 64) m = fmaxf(m, io.part_ml[(int64_t)p * io.rows + row].x);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  } else {
    for (int p = 0; p < parts; ++p) m = fmaxf(m, io.part_ml[(int64_t)p * io.rows + row].x);
  }
  float l = 0.f;
  float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int p = ALL ? g : 0; p < parts; p += side) {
    const int64_t prow = (int64_t)p * io.rows + row;
    const float2 ml = io.part_ml[prow];
    const float4 a = *reinterpret_cast<const float4*>(io.part_o + prow * D + 4 * c);
    const bool none = ml.y == 0.f;
    const float f = __builtin_amdgcn_exp2f(ml.x - m);
    l += none ? 0.f : ml.y * f;
    r.x += none ? 0.f : a.x * f;
    r.y += none ? 0.f : a.y * f;
    r.z += none ? 0.f : a.z * f;
    r.w += none ? 0.f : a.w * f;
  }
  if constexpr (ALL) {
    sums[g][c] = r;
    if (c == 0) ls[g] = l;
    __syncthreads();
    if (g > 0) return;
    l = 0.f;
    r = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      l += ls[i];
      r.x += sums[i][c].x;
      r.y += sums[i][c].y;
      r.z += sums[i][c].z;
      r.w += sums[i][c].w;
    }
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  uint2 w;
  w.x = pack_bf16x2(r.x * inv, r.y * inv);
  w.y = pack_bf16x2(r.z * inv, r.w * inv);
  *reinterpret_cast<uint2*>(io.o + (int64_t)row * D + 4 * c) = w;
  if (io.lse && c == 0) io.lse[row] = lse_of(m, l);
}

template <int D>
hipError_t join_parts(const Q8IO& io, int32_t parts, int num_cu, hipStream_t stream) {
  constexpr int P = 1024 / D;  // rows of a workgroup, or threads of a row's channel group
  if (io.rows <= 8 * num_cu || parts > 8) hipLaunchKernelGGL((join_parts_kernel<D, true>), dim3(io.rows), dim3(256), 0, stream, io, parts);
  else hipLaunchKernelGGL((join_parts_kernel<D, false>), dim3((io.rows + P - 1) / P), dim3(256), 0, stream, io, parts);
  return hipGetLastError();
}

// The form of a dense call: waves of 32 rows in a workgroup (0: the kernel for few rows, 32 rows a
// workgroup) and sets of them that share its keys, slabs of rows, parts of the keys.
struct DenseQ8Plan {
  int waves, sets;
  int32_t slabs, parts;
};

// Expected time of a form, in us. With m workgroups on the busiest CU, which share it: f0 + f m
// for starting and storing, and for every 64 keys of a part a + c m; at least what the codes
// take at 5 TB/s, more where CUs idle in the last round and where few workgroups leave a tail.
// Parts cost a second launch, some time each and their way through memory. f, a and c are fits to 256 m
// workgroups, m = 1 .. 6, of 512 and 4608 keys and to the scales of an image; measured at d =
// 128, us by the forms with few, 4 and 8 waves: 2 x 16 heads, 256 x 521 keys 9.1 / 15.6 / 22.5,
// 400 x 921 16.8 / 21.7 / 31.4, 1024 x 2521 64 / 49.6 / 70, 1600 x 4121 158 / 119.7 / 115.2,
// 2304 x 6425 314 / 277 / 342, 4096 x 10521 - / 612 / 592; 8 heads, 1024 x 2521 21.3 / 46.8 /
// 70. Sets are for launches of up to a workgroup a CU, which then has two waves a SIMD, and for no
// larger ones, where the other forms beat their estimate (d = 128, by four sets of two and by
// what is taken now: 2304 x 6425, 2 x 16 heads 329 / 281, 8 heads 178 / 157, 2 x 12 heads, 1600 x
// 4121 123 / 105; d = 64, 12 heads, 4096 x 10521 184 / 190). Two sets of four waves against one:
// 256 workgroups of 10521 keys 160 / 174 (d = 64 104 / 124), 192 of 5575 80.5 / 95, 256 of 2521
// 46.0 / 49.6; 384 workgroups 297 / 282. Four sets of two against the best of the others: d = 64,
// 16 heads, 646 x 2755 20.3 / 22.9, 1024 x 2521 19.7 / 22.6, d = 128, 12 heads, 1024 x 2521 28.2 /
// 30.8; 8 heads, 1024 x 2521 28.0 / 21; without a workspace, 4 heads, 4096 x 10521 96.6 / 114 (90
// in four parts of the others). One token of 8 heads, 10521 keys of one head: 281 us in one part,
// 11.5 in 21, 13.7 in 83; one token of 4 x 32 heads, up to 42521 keys of 8 heads:
// 76.8 in 8 parts, 58.4 in 16, 62.2 in 32.
struct DenseForm {
  int waves, sets;
  float f0, f, a, c;
};
constexpr DenseForm kDenseForms[2][5] = {
    // d = 64, d = 128
    {{0, 1, 3.f, .6f, .05f, .20f}, {2, 4, 2.5f, 3.f, 0.f, 1.38f}, {4, 1, 3.f, 1.3f, .2f, .53f}, {4, 2, 4.5f, 4.4f, 0.f, 1.15f},
     {8, 1, 4.f, 4.4f, 0.f, 1.12f}},
    {{0, 1, 2.f, 2.2f, .15f, .35f}, {2, 4, 5.f, 4.5f, 0.f, 1.92f}, {4, 1, 3.5f, 3.f, .3f, .92f}, {4, 2, 5.5f, 6.f, 0.f, 1.8f},
     {8, 1, 5.f, 6.f, 0.f, 1.77f}}};
constexpr int kMostParts = 128;

DenseQ8Plan dense_plan(int32_t planes, int32_t group, int32_t n_q, int32_t n_kv, int32_t d, int num_cu, bool may_split) {
  const int64_t rows = (int64_t)group * n_q, chunks = ((int64_t)n_kv + 63) / 64;
  const float memory = (float)planes * n_kv * d * (2.f / 5e6f);
  DenseQ8Plan best{0, 1, 1, 1};
  float best_us = INFINITY;
  for (const DenseForm& f : kDenseForms[d == 128]) {
    const int64_t per = f.waves ? 32 * f.waves : 32, slabs = (rows + per - 1) / per, items = planes * slabs;
    auto consider = [&](int64_t parts) {
      if (f.sets > 1 && items > num_cu) return;
      if (parts > 1 && (!may_split || f.sets > 1 || parts > chunks || parts > kMostParts)) return;
      const float m = (float)((items * parts + num_cu - 1) / num_cu), even = (float)(items * parts) / (float)num_cu;
      const float walk = (float)((chunks + parts * f.sets - 1) / (parts * f.sets)) * (f.a + f.c * m);
      const float read = memory * (m / even) * (1.f + .25f / m);
      float us = f.f0 + f.f * m + (walk > read ? walk : read);
      if (parts > 1) us += 3.f + .08f * parts + (float)parts * planes * rows * d * (8.f / 6e6f);
      if (us < best_us) {
        best_us = us;
        best = DenseQ8Plan{f.waves, f.sets, (int32_t)slabs, (int32_t)parts};
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

int32_t padded_grid(const Q8IO& io) { return io.swizzle ? (io.n_items + 7) / 8 * 8 : io.n_items; }

template <int D, int QW, int KS, class Src>
hipError_t launch_one(const Q8IO& io, const Src& src, hipStream_t stream) {
  hipLaunchKernelGGL((attn_q8_kernel<D, QW, KS, Src>), dim3(padded_grid(io)), dim3(QW * KS * 64), 0, stream, io, src);
  return hipGetLastError();
}

int64_t part_floats(int32_t parts, int64_t rows, int32_t d) { return (int64_t)parts * rows * (d + 2); }

}  // namespace

int64_t dense_q8_workspace(int32_t B, int32_t H, int32_t H_kv, int32_t n_q, int32_t n_kv, int32_t d, int num_cu) {
  const DenseQ8Plan p = dense_plan(B * H_kv, H / H_kv, n_q, n_kv, d, num_cu, true);
  return p.parts > 1 ? 4 * part_floats(p.parts, (int64_t)B * H * n_q, d) : 0;
}

Q8Form dense_q8_form(int32_t B, int32_t H, int32_t H_kv, int32_t n_q, int32_t n_kv, int32_t d, int num_cu, bool workspace) {
  const DenseQ8Plan p = dense_plan(B * H_kv, H / H_kv, n_q, n_kv, d, num_cu, workspace);
  return Q8Form{p.waves, p.sets, p.parts};
}

hipError_t launch_dense_attn_q8(const DenseQ8Args& a, hipStream_t stream) {
  const int32_t group = a.H / a.H_kv;
  const DenseQ8Plan p = dense_plan(a.B * a.H_kv, group, a.n_q, a.n_kv, a.d, a.num_cu, a.workspace != nullptr);
  Q8IO io;
  io.q = static_cast<const bf16_bits*>(a.q);
  io.o = static_cast<bf16_bits*>(a.o);
  io.lse = a.lse;
  io.q_bh_stride = a.q_bh_stride;
  io.c = a.c8;
  io.o_rows = a.n_q;
  io.n_items = a.B * a.H_kv * p.slabs * p.parts;
  io.swizzle = a.swizzle;
  io.scale_log2 = a.softmax_scale * kLog2e;
  io.rows = a.B * a.H * a.n_q;
  io.part_o = p.parts > 1 ? a.workspace : nullptr;
  io.part_ml = p.parts > 1 ? reinterpret_cast<float2*>(a.workspace + (int64_t)p.parts * io.rows * a.d) : nullptr;
  auto fill = [&](auto src) {
    src.n_q = a.n_q;
    src.n_kv = a.n_kv;
    src.H_kv = a.H_kv;
    src.group = group;
    src.slabs = p.slabs;
    src.q_per_wg = p.waves ? 32 * p.waves : 32;
    src.parts = p.parts;
    src.kv_len = a.kv_len;
    return src;
  };
  hipError_t e = hipErrorInvalidValue;
  if (p.waves == 0) {
    const int32_t grid = padded_grid(io);
    const DenseQ8Src<32> src = fill(DenseQ8Src<32>{});
    if (a.d == 128) hipLaunchKernelGGL((attn_q8_rows_kernel<128>), dim3(grid), dim3(kRowWaves * 64), 0, stream, io, src);
    else hipLaunchKernelGGL((attn_q8_rows_kernel<64>), dim3(grid), dim3(kRowWaves * 64), 0, stream, io, src);
    e = hipGetLastError();
  } else {
    const DenseQ8Src<64> src = fill(DenseQ8Src<64>{});
#define SV_DENSE(DD, NN, KK) \
  if (a.d == DD && p.waves == NN && p.sets == KK) e = launch_one<DD, NN, KK>(io, src, stream);
    SV_DENSE(64, 2, 4) SV_DENSE(64, 4, 1) SV_DENSE(64, 4, 2) SV_DENSE(64, 8, 1)
    SV_DENSE(128, 2, 4) SV_DENSE(128, 4, 1) SV_DENSE(128, 4, 2) SV_DENSE(128, 8, 1)
#undef SV_DENSE
  }
  if (e != hipSuccess || p.parts == 1) return e;
  return a.d == 128 ? join_parts<128>(io, p.parts, a.num_cu, stream) : join_parts<64>(io, p.parts, a.num_cu, stream);
}

Q8Form sparse_q8_form(const GeoTable& G, int32_t k, int32_t BH, int32_t d, int num_cu) {
  const int32_t tile_q = G.eh[k - 1] * G.ew[k - 1];
  const int nw = waves_for(tile_q);
  const int32_t items = BH * tiles_of(G, k) * ((tile_q + nw * kQPerWave - 1) / (nw * kQPerWave));
  // Tiles of 33 to 64 queries (8 x 8): launches of few waves a SIMD walk their rows in two parts
  // (64 x 64 scale, d = 128: 512 workgroups 39.0 us against 50.7, 640 57.0 / 53.6; d = 64: 512
  // 27.5 / 38.4, 768 33.9 / 39.7, 896 44.1 / 42.3; past that within 8% of each other, with the
  // rounds that either makes), up to one workgroup a CU in four, where the cache is long enough
  // for rows that give back what the join costs (256 workgroups, 10521 tokens: d = 128 26.9 in
  // four against 29.4, d = 64 18.8 / 21.1; 921 tokens 20.9 / 21.1 and 14.2 / 15.1; 521 17.4 /
  // 16.3 and 12.2 / 12.0; past one workgroup a CU, 320: 47.6 / 38.1 and 32.9 / 26.6).
  int32_t sets = 1;
  if (nw == 2 && items <= (d == 64 ? 3 : 2) * num_cu) sets = items <= num_cu && G.C[k] >= 640 ? 4 : 2;
  return Q8Form{nw, sets, 1};
}

hipError_t launch_sparse_attn_q8(const SparseQ8Args& a, hipStream_t stream) {
  const GeoTable& G = *a.G;
  const int32_t tile_q = G.eh[a.k - 1] * G.ew[a.k - 1], G_k = tiles_of(G, a.k);
  const Q8Form form = sparse_q8_form(G, a.k, a.BH, a.d, a.num_cu);
  const int nw = form.waves;
  const int32_t qpw = nw * kQPerWave, slabs = (tile_q + qpw - 1) / qpw;
  Q8IO io;
  io.q = static_cast<const bf16_bits*>(a.q);
  io.o = static_cast<bf16_bits*>(a.o);
  io.lse = a.lse;
  io.q_bh_stride = a.q_bh_stride;
  io.c = a.c8;
  io.o_rows = G.h[a.k - 1] * G.w[a.k - 1];
  io.n_items = a.BH * G_k * slabs;
  io.swizzle = a.swizzle;
  io.scale_log2 = a.softmax_scale * kLog2e;
  io.part_o = nullptr;
  io.part_ml = nullptr;
  io.rows = a.BH * io.o_rows;
  SparseQ8Src src;
  src.group = a.H / a.H_kv;
  src.max_chunks_per_block = 0;  // (of the block tables, which these kernels do not use)
  src.G = G;
  src.row_ptr = a.row_ptr;
  src.col_idx = a.col_idx;
  src.schedule = a.schedule;
  src.k = a.k;
  src.G_k = G_k;
  src.q_per_wg = qpw;
  src.slabs = slabs;
  src.n_rows = a.BH * G_k;
  const int ks = form.sets;
#define SV_SPARSE(DD, NN, KK) \
  if (a.d == DD && nw == NN && ks == KK) return launch_one<DD, NN, KK>(io, src, stream);
  SV_SPARSE(64, 1, 1) SV_SPARSE(64, 2, 1) SV_SPARSE(64, 2, 2) SV_SPARSE(64, 2, 4) SV_SPARSE(64, 4, 1) SV_SPARSE(64, 8, 1)
  SV_SPARSE(128, 1, 1) SV_SPARSE(128, 2, 1) SV_SPARSE(128, 2, 2) SV_SPARSE(128, 2, 4) SV_SPARSE(128, 4, 1) SV_SPARSE(128, 8, 1)
#undef SV_SPARSE
  return hipErrorInvalidValue;
}

}  // namespace sparvar
