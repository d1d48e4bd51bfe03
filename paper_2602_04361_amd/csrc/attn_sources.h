// What an attention workgroup walks: its queries (QuerySet) and the key chunks of its
// source, a slab of a dense call, a CSR row of 2-D blocks or a group of neighbouring
// rows, a row of listed tokens, or a row of 1-D blocks.
#pragma once

#include <type_traits>

#include "device_common.h"

namespace sparvar {

// Queries of one workgroup: slot i in [q0, q1) is plane row
// qbase + (i / qnc) * qstride + i % qnc.
struct QuerySet {
  int32_t bh, qbase, qnc, qstride, q0, q1;
};

// ---------------------------------------------------------------- key sources
template <int KC>
struct DenseCursor {
  int32_t pos, n;
  __device__ __forceinline__ bool next(Chunk& c) {
    if (pos >= n) return false;
    const int32_t cnt = (n - pos < KC) ? n - pos : KC;
    c = run_chunk(pos, cnt);
    pos += cnt;
    return true;
  }
};

template <int KC>
struct DenseSrc {
  static constexpr bool kSparse = false;
  static constexpr bool kGrouped = false;
  static constexpr bool kTokens = false;
  int32_t n_q, n_kv, slabs, q_per_wg;
  template <int NT>
  static constexpr int table_bytes() { return 16; }
  __device__ __forceinline__ int tile_of(int) const { return 0; }
  __device__ __forceinline__ QuerySet queries(int32_t item, int wave) const {
    QuerySet s;
    s.bh = item / slabs;
    const int32_t slab = item - s.bh * slabs;
    s.qbase = 0;
    s.qnc = n_q;
    s.qstride = 0;
    const int32_t q0 = slab * q_per_wg;
    s.q1 = (q0 + q_per_wg < n_q) ? q0 + q_per_wg : n_q;
    s.q0 = q0 + wave * kQPerWave;
    return s;
  }
  __device__ __forceinline__ DenseCursor<KC> cursor(int32_t) const { return DenseCursor<KC>{0, n_kv}; }
};

// Restricts a dense cursor to split s of ks; returns the chunks of the longest split.
template <int KC>
__device__ __forceinline__ int32_t take_split(DenseCursor<KC>& c, int s, int ks) {
  const int32_t per = ((c.n + KC - 1) / KC + ks - 1) / ks;
  c.pos = s * per * KC;
  c.n = c.pos + per * KC < c.n ? c.pos + per * KC : c.n;
  return per;
}

// Key tokens listed one by one (token-granular rows): chunk slot r holds the
// token tokens[base + r].
template <int KC>
struct TokenCursor {
  int32_t pos, len, row_off;
  __device__ __forceinline__ bool next(Chunk& c) {
    if (pos >= len) return false;
    const int32_t cnt = (len - pos < KC) ? len - pos : KC;
    c = run_chunk(row_off + pos, cnt);
    pos += cnt;
    return true;
  }
};

// Rows of key tokens for 1-D query blocks of C contiguous queries (C = 32 NW):
// row r = (b*H + h) * n_blocks + g lists, for the queries [g C, g C + C) of the
// plane, ascending token ids in [0, n_kv) followed by padding (any id outside
// that range), at a fixed stride M.
template <int KC>
struct TokenSrc {
  static constexpr bool kSparse = false;
  static constexpr bool kGrouped = false;
  static constexpr bool kTokens = true;
  const int32_t* tokens;
  int32_t M, C, n_q, n_kv, n_blocks;
  template <int NT>
  static constexpr int table_bytes() { return 64; }
  __device__ __forceinline__ int tile_of(int) const { return 0; }
  __device__ __forceinline__ QuerySet queries(int32_t item, int wave) const {
    QuerySet s;
    s.bh = item / n_blocks;
    const int32_t g = item - s.bh * n_blocks;
    s.qbase = g * C;
    s.qnc = 1 << 30;  // contiguous rows
    s.qstride = 0;
    s.q0 = wave * kQPerWave;
    s.q1 = (n_q - g * C < C) ? n_q - g * C : C;
    return s;
  }
  // The row's token count (its ids up to the first padding entry), by the whole workgroup.
  template <int NT>
  __device__ __forceinline__ TokenCursor<KC> token_cursor(int32_t item, char* lds) const {
    const int32_t* row = tokens + (int64_t)item * M;
    int32_t cnt = 0;
    for (int32_t i = threadIdx.x; i < M; i += NT) {
      const int32_t t = row[i];
      cnt += (t >= 0 && t < n_kv) ? 1 : 0;
    }
    int32_t total;
    block_excl_scan<NT>(cnt, reinterpret_cast<int32_t*>(lds), total);
    TokenCursor<KC> c;
    c.pos = 0;
    c.len = __builtin_amdgcn_readfirstlane(total);
    c.row_off = item * M;
    return c;
  }
};

// Restricts a token cursor to split s of ks; returns the chunks of the longest split.
template <int KC>
__device__ __forceinline__ int32_t take_split(TokenCursor<KC>& c, int s, int ks) {
  const int32_t per = ((c.len + KC - 1) / KC + ks - 1) / ks;
  c.pos = s * per * KC;
  c.len = c.pos + per * KC < c.len ? c.pos + per * KC : c.len;
  return per;
}

// Listed 1-D key blocks of B contiguous tokens: consecutive ids are merged into
// one run of the cache, cut into chunks of at most KC keys. The first kRunTable
// entries of the row are staged in LDS; later ones are read from global memory.
// The walk ends at the first id outside [0, nkb).
constexpr int kRunTable = 512;

template <int KC>
struct RunCursor {
  const int32_t* ids;  // LDS
  const int32_t* row;  // global
  int32_t pos, len, B, n_kv, nkb, run_base, run_left;
  __device__ __forceinline__ int32_t id_at(int32_t p) const {
    return __builtin_amdgcn_readfirstlane(p < kRunTable ? ids[p] : row[p]);
  }
  __device__ __forceinline__ bool next(Chunk& c) {
    if (run_left == 0) {
      if (pos >= len) return false;
      int32_t v = id_at(pos);
      if ((uint32_t)v >= (uint32_t)nkb) {
        pos = len;
        return false;
      }
      ++pos;
      run_base = v * B;
      while (pos < len && id_at(pos) == v + 1) {
        ++v;
        ++pos;
      }
      const int32_t end = v * B + B;
      run_left = (end < n_kv ? end : n_kv) - run_base;
    }
    const int32_t cnt = run_left < KC ? run_left : KC;
    c = run_chunk(run_base, cnt);
    run_base += cnt;
    run_left -= cnt;
    return true;
  }
};

// Restricts a run cursor to split s of ks (whole listed blocks: B is a multiple of
// KC, so a block is B / KC chunks but for the cache's last); returns the chunks of
// the longest split. Counts the row's ids up to the first one out of range.
template <int KC>
__device__ __forceinline__ int32_t take_split(RunCursor<KC>& c, int s, int ks) {
  int32_t n = 0;
  for (int32_t p0 = 0; p0 < c.len; p0 += 64) {
    const int32_t p = p0 + (int32_t)(threadIdx.x & 63);
    const int32_t v = p < c.len ? (p < kRunTable ? c.ids[p] : c.row[p]) : -1;
    const uint64_t out = ~__builtin_amdgcn_ballot_w64((uint32_t)v < (uint32_t)c.nkb);
    if (out) {
      n = p0 + __builtin_ctzll(out);
      break;
    }
    n = p0 + 64;
  }
  n = n < c.len ? n : c.len;
  const int32_t per = (n + ks - 1) / ks;
  c.pos = s * per;
  c.len = c.pos + per < n ? c.pos + per : n;
  return per * ((c.B + KC - 1) / KC);
}

// 1-D query blocks of C = 32 NW contiguous queries, each with a row of 1-D key
// blocks of C tokens (the CSLA block mask). Row g of rows, shared by every
// (b, h), lists ascending ids in [0, ceil(n_kv / C)) followed by padding (any id
// outside that range), at a fixed stride M.
template <int KC>
struct BlockRowSrc {
  static constexpr bool kSparse = false;
  static constexpr bool kGrouped = false;
  static constexpr bool kTokens = false;
  static constexpr bool kRuns = true;
  const int32_t* rows;
  int32_t M, C, n_q, n_kv, n_blocks;
  template <int NT>
  static constexpr int table_bytes() { return 4 * kRunTable; }
  __device__ __forceinline__ int tile_of(int) const { return 0; }
  __device__ __forceinline__ QuerySet queries(int32_t item, int wave) const {
    QuerySet s;
    s.bh = item / n_blocks;
    const int32_t g = item - s.bh * n_blocks;
    s.qbase = g * C;
    s.qnc = 1 << 30;  // contiguous rows
    s.qstride = 0;
    s.q0 = wave * kQPerWave;
    s.q1 = (n_q - g * C < C) ? n_q - g * C : C;
    return s;
  }
  // Stages the head of the row in LDS, by the whole workgroup.
  template <int NT>
  __device__ __forceinline__ RunCursor<KC> run_cursor(int32_t item, char* lds) const {
    const int32_t g = item % n_blocks;
    const int32_t* row = rows + (int64_t)g * M;
    int32_t* ids = reinterpret_cast<int32_t*>(lds);
    const int32_t lim = M < kRunTable ? M : kRunTable;
    for (int32_t i = threadIdx.x; i < lim; i += NT) ids[i] = row[i];
    __syncthreads();
    RunCursor<KC> c;
    c.ids = ids;
    c.row = row;
    c.pos = 0;
    c.len = M;
    c.B = C;
    c.n_kv = n_kv;
    c.nkb = (n_kv + C - 1) / C;
    c.run_base = 0;
    c.run_left = 0;
    return c;
  }
};

// Walks the kept blocks of one CSR row as chunks of at most KC keys.
// Consecutive blocks whose tokens are contiguous in the cache (whole small
// scales such as the sink scales) are merged into one run and cut at KC;
// other tiles are emitted as bands of whole tile rows (or row pieces when a
// tile row is longer than KC).
template <int KC>
struct CsrCursor {
  const GeoTable* G;
  const int32_t* __restrict__ col;
  int32_t pos, end, nb;
  int32_t run_base, run_left;
  Tile t;
  int32_t t_row, t_col;

  __device__ __forceinline__ bool fetch(int32_t& v) {
    while (pos < end) {
      v = col[pos++];
      if (v >= 0 && v < nb) return true;
    }
    return false;
  }

  __device__ __forceinline__ static bool contiguous(const Tile& x) { return x.nr == 1 || x.nc == x.stride; }

  __device__ __forceinline__ bool next(Chunk& c) {
    for (;;) {
      if (run_left > 0) {
        const int32_t n = run_left < KC ? run_left : KC;
        c = run_chunk(run_base, n);
        run_base += n;
        run_left -= n;
        return true;
      }
      if (t_row < t.nr) {
        if (t.nc <= KC) {
          const int32_t rpc = KC / t.nc;
          const int32_t rows = (t.nr - t_row < rpc) ? t.nr - t_row : rpc;
          c = make_chunk(t.base + t_row * t.stride, t.nc, t.stride, rows * t.nc);
          t_row += rows;
        } else {
          const int32_t n = (t.nc - t_col < KC) ? t.nc - t_col : KC;
          c = run_chunk(t.base + t_row * t.stride + t_col, n);
          t_col += n;
          if (t_col >= t.nc) {
            t_col = 0;
            ++t_row;
          }
        }
        return true;
      }
      int32_t v;
      if (!fetch(v)) return false;
      const Tile x = block_tile(*G, v);
      if (contiguous(x)) {
        run_base = x.base;
        run_left = x.nr * x.nc;
        while (pos < end) {
          const int32_t v2 = col[pos];
          if (v2 < 0 || v2 >= nb) break;
          const Tile y = block_tile(*G, v2);
          if (!contiguous(y) || y.base != run_base + run_left) break;
          run_left += y.nr * y.nc;
          ++pos;
        }
      } else {
        t = x;
        t_row = 0;
        t_col = 0;
      }
    }
  }
};

// Chunk list of a block list, decoded in parallel by the whole workgroup into an
// LDS table: each refill decodes up to `group` blocks (one per thread), merges
// runs of contiguous blocks that have the same tile mask, splits everything into
// chunks of at most KC keys and writes 8-byte descriptors plus the mask; the main
// loop then only reads descriptors. Descriptor: x = first token,
// y = stride << 16 | nc << 8 | count; in the mask word the tile mask << 24 (a group
// has at most 8 tiles) | ceil(65536 / nc), so that a step needs no table lookup of it.
// Blocks supplies the ids: id(i) and mask(i) for i in the current segment
// [pos, end), and segment(pos, end), which moves to the next segment (false when
// there is none). fill() is a call of the whole workgroup; next() one of a wave, and
// under key splits each split's waves walk their own part of the table.
constexpr int kTableCap = 256;

template <int NT>
struct TableLds {  // byte offsets inside the table region
  static constexpr int kTbl = 0;
  static constexpr int kTmask = kTbl + kTableCap * 8;
  static constexpr int kInfo = kTmask + kTableCap * 4;
  static constexpr int kImask = kInfo + NT * 16;
  static constexpr int kWt = kImask + NT * 4;
  static constexpr int kGeo = kWt + 16 * 4;  // LDS copy of the geometry table
  static constexpr int kBytes = kGeo + (int)((sizeof(GeoTable) + 15) / 16 * 16);
};

// Copies the geometry table from the kernel arguments into LDS, where the
// per-thread block decode of a refill reads it: indexed per lane, the
// kernel-argument copy is read with a chain of dependent global loads (one per
// scale searched), which made the first refill of every workgroup take
// microseconds. Visible after the next workgroup barrier.
template <int NT>
__device__ __forceinline__ const GeoTable* stage_geometry(const GeoTable& G, char* lds) {
  static_assert(sizeof(GeoTable) % 4 == 0, "geometry table is 32-bit words");
  constexpr int kWords = (int)(sizeof(GeoTable) / 4);
  const int32_t* s = reinterpret_cast<const int32_t*>(&G);
  int32_t* d = reinterpret_cast<int32_t*>(lds + TableLds<NT>::kGeo);
  for (int i = threadIdx.x; i < kWords; i += NT) d[i] = s[i];
  return reinterpret_cast<const GeoTable*>(lds + TableLds<NT>::kGeo);
}

template <int KC, int NT, class Blocks>
struct TableCursor {
  const GeoTable* G;
  Blocks blocks;
  int32_t nb, group;
  int32_t pos, end;  // entries of the current segment not yet decoded
  int32_t tn, ti;    // table fill and read position
  char* lds;         // TableLds<NT> region

  __device__ __forceinline__ static bool contiguous(const int4& x) { return x.y == 1 || x.z == x.w; }

  __device__ static int32_t chunks_of(const int4& x, int32_t total_if_run) {
    if (contiguous(x)) return (total_if_run + KC - 1) / KC;
    if (x.z <= KC) {
      const int32_t rpc = KC / x.z;
      return (x.y + rpc - 1) / rpc;
    }
    return x.y * ((x.z + KC - 1) / KC);
  }

  __device__ __forceinline__ void refill() {
    using L = TableLds<NT>;
    uint2* tbl = reinterpret_cast<uint2*>(lds + L::kTbl);
    uint32_t* tmask = reinterpret_cast<uint32_t*>(lds + L::kTmask);
    int4* info = reinterpret_cast<int4*>(lds + L::kInfo);
    uint32_t* imask = reinterpret_cast<uint32_t*>(lds + L::kImask);
    int32_t* wt = reinterpret_cast<int32_t*>(lds + L::kWt);
    const int tid = fresh_tid();
    __syncthreads();
    const int32_t nblk = (end - pos < group) ? end - pos : group;
    if (tid < nblk) {
      const int32_t v = blocks.id(pos + tid);
      int4 x = make_int4(0, 0, 1, 1);
      if (v >= 0 && v < nb) {
        const Tile t = block_tile(*G, v);
        x = make_int4(t.base, t.nr, t.nc, t.stride);
      }
      info[tid] = x;
      imask[tid] = blocks.mask(pos + tid);
    }
    __syncthreads();
    int32_t n = 0, run_total = 0;
    int4 x = make_int4(0, 0, 1, 1);
    uint32_t m = 0;
    if (tid < nblk) {
      x = info[tid];
      m = imask[tid];
      if (x.y > 0) {
        bool cont = false;
        if (contiguous(x) && tid > 0) {
          const int4 p = info[tid - 1];
          cont = p.y > 0 && contiguous(p) && p.x + p.y * p.z == x.x && imask[tid - 1] == m;
        }
        if (!cont) {
          run_total = x.y * x.z;
          if (contiguous(x)) {
            for (int32_t u = tid + 1; u < nblk; ++u) {
              const int4 y = info[u];
              if (y.y > 0 && contiguous(y) && y.x == x.x + run_total && imask[u] == m) run_total += y.y * y.z;
              else break;
            }
          }
          n = chunks_of(x, run_total);
        }
      }
    }
    int32_t total;
    int32_t o = block_excl_scan<NT>(n, wt, total);
    if (n > 0) {
      if (contiguous(x)) {
        for (int32_t done = 0; done < run_total; done += KC, ++o) {
          const int32_t cnt = (run_total - done < KC) ? run_total - done : KC;
          tbl[o] = make_uint2((uint32_t)(x.x + done), (uint32_t)((kChunk << 16) | (kChunk << 8) | cnt));
          tmask[o] = m << 24 | 65536 / kChunk;
        }
      } else if (x.z <= KC) {
        const int32_t rpc = KC / x.z;
        const uint32_t magic = 65535u / (uint32_t)x.z + 1;
        for (int32_t r0 = 0; r0 < x.y; r0 += rpc, ++o) {
          const int32_t rows = (x.y - r0 < rpc) ? x.y - r0 : rpc;
          tbl[o] = make_uint2((uint32_t)(x.x + r0 * x.w), (uint32_t)((x.w << 16) | (x.z << 8) | (rows * x.z)));
          tmask[o] = m << 24 | magic;
        }
      } else {
        for (int32_t r0 = 0; r0 < x.y; ++r0)
          for (int32_t c0 = 0; c0 < x.z; c0 += KC, ++o) {
            const int32_t cnt = (x.z - c0 < KC) ? x.z - c0 : KC;
            tbl[o] = make_uint2((uint32_t)(x.x + r0 * x.w + c0), (uint32_t)((kChunk << 16) | (kChunk << 8) | cnt));
            tmask[o] = m << 24 | 65536 / kChunk;
          }
      }
    }
    __syncthreads();
    tn = __builtin_amdgcn_readfirstlane(total);
    ti = 0;
    pos += nblk;
  }

  // Decodes the next part of the list into the table (false: none left). Called by
  // the whole workgroup between two walks of the table, never inside one: decoding
  // inside the walk put its registers and code into every pipeline step.
  __device__ __forceinline__ bool fill() {
    do {
      while (pos >= end)
        if (!blocks.segment(pos, end)) return false;
      refill();
    } while (tn == 0);
    return true;
  }

  // Restricts the walk of the filled table to split s of ks; returns the chunks of the longest split.
  __device__ __forceinline__ int32_t take_split(int s, int ks) {
    const int32_t per = (tn + ks - 1) / ks;
    ti = s * per;
    tn = ti + per < tn ? ti + per : tn;
    return per;
  }

  // Whether another fill() may find something (most lists fit one table).
  __device__ __forceinline__ bool more() const { return pos < end || blocks.more(); }

  __device__ __forceinline__ bool next(Chunk& c) {
    using L = TableLds<NT>;
    if (ti >= tn) return false;
    const uint2 e = reinterpret_cast<const uint2*>(lds + L::kTbl)[ti];
    const uint32_t m = reinterpret_cast<const uint32_t*>(lds + L::kTmask)[ti];
    ++ti;
    const uint32_t y = __builtin_amdgcn_readfirstlane(e.y);
    const uint32_t z = __builtin_amdgcn_readfirstlane(m);
    c.base = __builtin_amdgcn_readfirstlane(e.x);
    c.stride = (int32_t)(y >> 16);
    c.nc = (int32_t)((y >> 8) & 0xff);
    c.count = (int32_t)(y & 0xff);
    c.magic = (int32_t)(z & 0x1ffff);
    c.mask = z >> 24;
    return true;
  }
};

// Block list of one CSR row in global memory (a single segment, every tile).
struct CsrBlocks {
  const int32_t* __restrict__ col;
  int32_t p0, p1;
  bool done;
  __device__ __forceinline__ int32_t id(int32_t i) const { return col[i]; }
  __device__ __forceinline__ uint32_t mask(int32_t) const { return 0xffu; }
  __device__ __forceinline__ bool more() const { return !done; }
  __device__ __forceinline__ bool segment(int32_t& pos, int32_t& end) {
    if (done) return false;
    done = true;
    pos = p0;
    end = p1;
    return true;
  }
};

template <int KC>
struct SparseSrc {
  static constexpr bool kSparse = true;
  static constexpr bool kGrouped = false;
  static constexpr bool kTokens = false;
  GeoTable G;
  const int32_t* row_ptr;
  const int32_t* col_idx;
  const int32_t* schedule;  // nullable launch order of rows; ignored when schedule[0] < 0 (an order of groups)
  int32_t k, G_k, slabs, q_per_wg, n_rows;
  int32_t max_chunks_per_block;  // bound used to size a table refill

  template <int NT>
  static constexpr int table_bytes() { return TableLds<NT>::kBytes; }
  __device__ __forceinline__ int tile_of(int) const { return 0; }
  __device__ __forceinline__ int32_t row_of(int32_t item) const {
    const int32_t r = item / slabs;
    if (!schedule || schedule[0] < 0) return r;
    const int32_t v = schedule[r];
    return (v >= 0 && v < n_rows) ? v : r;
  }
  __device__ __forceinline__ QuerySet queries(int32_t item, int wave) const {
    const int32_t r = row_of(item);
    const int32_t slab = item - (item / slabs) * slabs;
    QuerySet s;
    s.bh = r / G_k;
    const int32_t g = r - s.bh * G_k;
    const int32_t tw = G.Tw[k - 1];
    const Tile t = tile_at(G, k, g / tw, g % tw);
    s.qbase = t.base - G.C[k - 1];  // row inside the scale-k query plane
    s.qnc = t.nc;
    s.qstride = t.stride;
    const int32_t nq = t.nr * t.nc;
    const int32_t q0 = slab * q_per_wg;
    s.q1 = (q0 + q_per_wg < nq) ? q0 + q_per_wg : nq;
    s.q0 = q0 + wave * kQPerWave;
    return s;
  }
  __device__ __forceinline__ CsrCursor<KC> cursor(int32_t item) const {
    const int32_t r = row_of(item);
    CsrCursor<KC> c;
    c.G = &G;
    c.col = col_idx;
    c.pos = row_ptr[r];
    c.end = row_ptr[r + 1];
    c.nb = G.NB[k];
    c.run_base = 0;
    c.run_left = 0;
    c.t.nr = 0;
    c.t_row = 0;
    c.t_col = 0;
    return c;
  }
  template <int NT>
  __device__ __forceinline__ TableCursor<KC, NT, CsrBlocks> table_cursor(int32_t item, char* lds) const {
    const int32_t r = row_of(item);
    TableCursor<KC, NT, CsrBlocks> c;
    c.G = stage_geometry<NT>(G, lds);  // the first refill starts with a barrier
    c.blocks.col = col_idx;
    c.blocks.p0 = row_ptr[r];
    c.blocks.p1 = row_ptr[r + 1];
    c.blocks.done = false;
    c.nb = G.NB[k];
    const int32_t g = kTableCap / (max_chunks_per_block > 0 ? max_chunks_per_block : 1);
    c.group = g < NT ? (g > 0 ? g : 1) : NT;
    c.pos = 0;
    c.end = 0;
    c.tn = 0;
    c.ti = 0;
    c.lds = lds;
    return c;
  }
};

// ------------------------------------------------------- grouped query tiles
// A workgroup serves a group of T neighbouring query tiles of scale k (T = 2,
// 4 or 8; gh x gw tiles) and walks the union of their CSR rows once: every
// staged chunk carries the mask of the group's tiles whose row lists the block,
// and the waves of the other tiles skip it. Each tile still attends to exactly
// its own blocks; the union only lets tiles share each HBM -> LDS copy.
//
// Union of sorted rows, built in parallel (thread = row entry): each row's
// valid ids are compacted; an entry is the owner of its id when no lower row and
// no earlier entry of its own row holds the id; its place in the union is the
// number of owners with smaller ids, found by a binary search in every other
// row; its mask has a bit for every row holding the id. Rows longer than
// NT / T entries are served tile by tile instead, in windows of NT entries.
template <int NT>
struct GroupLds {
  static constexpr int kIds = 0;
  static constexpr int kOwnp = kIds + NT * 4;
  static constexpr int kUid = kOwnp + NT * 4;
  static constexpr int kUmask = kUid + NT * 4;
  static constexpr int kRowP = kUmask + NT * 4;
  static constexpr int kRowN = kRowP + 8 * 4;
  static constexpr int kRowC = kRowN + 8 * 4;
  static constexpr int kWt = kRowC + 8 * 4;
  static constexpr int kBytes = kWt + 16 * 4;
};

template <int NT>
struct GroupBlocks {
  static constexpr int kLgNT = NT == 512 ? 9 : NT == 256 ? 8 : NT == 128 ? 7 : 6;
  const int32_t* __restrict__ col;
  int32_t nb, T, lgT;
  bool by_tile, started;
  int32_t seg_t, seg_off;  // next window of the tile-by-tile mode
  char* lds;               // GroupLds<NT> region

  __device__ __forceinline__ int32_t* arr(int off) const { return reinterpret_cast<int32_t*>(lds + off); }
  __device__ __forceinline__ int32_t id(int32_t i) const { return arr(GroupLds<NT>::kUid)[i]; }
  __device__ __forceinline__ uint32_t mask(int32_t i) const {
    return (uint32_t)arr(GroupLds<NT>::kUmask)[i];
  }

  __device__ __forceinline__ bool more() const { return by_tile ? seg_t < T : !started; }

  __device__ __forceinline__ int32_t build_union() {
    using L = GroupLds<NT>;
    int32_t* ids = arr(L::kIds);
    int32_t* ownp = arr(L::kOwnp);
    const int32_t* rowp = arr(L::kRowP);
    const int32_t* rown = arr(L::kRowN);
    int32_t* rowc = arr(L::kRowC);
    int32_t* wt = arr(L::kWt);
    const int tid = fresh_tid();
    const int lgRC = kLgNT - lgT;
    const int32_t RC = 1 << lgRC;
    const int t = tid >> lgRC;
    const int32_t i = tid & (RC - 1);
    int32_t raw = -1;
    if (i < rown[t]) raw = col[rowp[t] + i];
    const bool valid = raw >= 0 && raw < nb;
    int32_t total;
    const int32_t e = block_excl_scan<NT>(valid ? 1 : 0, wt, total);
    ownp[tid] = e;
    __syncthreads();
    const int32_t row0 = ownp[t * RC];
    if (valid) ids[t * RC + (e - row0)] = raw;
    if (i == 0) rowc[t] = ((t + 1) * RC < NT ? ownp[(t + 1) * RC] : total) - row0;
    __syncthreads();

    const int32_t nt = rowc[t];
    int32_t v = 0;
    uint32_t m = 0;
    bool own = false;
    if (i < nt) {
      v = ids[t * RC + i];
      own = !(i > 0 && ids[t * RC + i - 1] == v);
      m = 1u << t;
    }
    int32_t lb[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      lb[u] = 0;
      if (u < T && i < nt) {
        if (u == t) {
          lb[u] = i;
        } else {
          const int32_t* r = ids + u * RC;
          const int32_t n = rowc[u];
          int32_t lo = 0, hi = n;
          while (lo < hi) {
            const int32_t mid = (lo + hi) >> 1;
            if (r[mid] < v) lo = mid + 1;
            else hi = mid;
          }
          lb[u] = lo;
          if (lo < n && r[lo] == v) {
            m |= 1u << u;
            if (u < t) own = false;
          }
        }
      }
    }
    int32_t owners;
    const int32_t e2 = block_excl_scan<NT>(own ? 1 : 0, wt, owners);
    ownp[tid] = e2;
    __syncthreads();
    if (own) {
      int32_t rank = 0;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        if (u < T) {
          const int32_t base = ownp[u * RC];
          const int32_t j = lb[u];
          const int32_t at = j < RC ? ownp[u * RC + j] : ((u + 1) * RC < NT ? ownp[(u + 1) * RC] : owners);
          rank += at - base;
        }
      }
      arr(L::kUid)[rank] = v;
      arr(L::kUmask)[rank] = (int32_t)m;
    }
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(owners);
  }

  __device__ __forceinline__ int32_t build_window() {
    using L = GroupLds<NT>;
    const int tid = fresh_tid();
    const int32_t n = arr(L::kRowN)[seg_t] - seg_off;
    int32_t raw = -1;
    if (tid < n) raw = col[arr(L::kRowP)[seg_t] + seg_off + tid];
    const bool valid = raw >= 0 && raw < nb;
    int32_t total;
    const int32_t e = block_excl_scan<NT>(valid ? 1 : 0, arr(L::kWt), total);
    if (valid) {
      arr(L::kUid)[e] = raw;
      arr(L::kUmask)[e] = 1 << seg_t;
    }
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(total);
  }

  __device__ __forceinline__ bool segment(int32_t& pos, int32_t& end) {
    if (!by_tile) {
      if (started) return false;
      started = true;
      end = build_union();
      pos = 0;
      return true;
    }
    const int32_t* rown = arr(GroupLds<NT>::kRowN);
    while (seg_t < T && seg_off >= rown[seg_t]) {
      ++seg_t;
      seg_off = 0;
    }
    if (seg_t >= T) return false;
    end = build_window();
    pos = 0;
    seg_off += NT;
    return true;
  }
};

template <int KC>
struct GroupSrc {
  static constexpr bool kSparse = true;
  static constexpr bool kGrouped = true;
  static constexpr bool kTokens = false;
  GeoTable G;
  const int32_t* row_ptr;
  const int32_t* col_idx;
  int32_t k, G_k;
  int32_t gh, gw, lgT;   // group of gh x gw tiles, T = gh * gw = 1 << lgT
  int32_t ngc, n_groups;  // groups per group row, groups per (b, h)
  uint32_t wave_tile, wave_slab;  // 4 bits per wave: the wave's tile in the group and its 32-query slab
  int32_t max_chunks_per_block;
  // Nullable launch order: order[p] = -2 - (group item launched at position p),
  // as the mapping call writes it; a row permutation (non-negative entries) is
  // not an order of groups and is ignored.
  const int32_t* order;
  static constexpr bool kRemap = true;

  __device__ __forceinline__ int32_t remap(int32_t p, int32_t n_items) const {
    if (!order || order[0] >= 0) return p;
    const int32_t v = -2 - order[p];
    return (v >= 0 && v < n_items) ? v : p;
  }

  template <int NT>
  static constexpr int table_bytes() { return TableLds<NT>::kBytes + GroupLds<NT>::kBytes; }
  __device__ __forceinline__ int tile_of(int wave) const { return (int)((wave_tile >> (4 * wave)) & 15u); }

  // Tile t of the group of item; false when it lies outside the scale.
  __device__ __forceinline__ bool group_tile(int32_t item, int t, int32_t& bh, int32_t& a, int32_t& c) const {
    bh = item / n_groups;
    const int32_t gi = item - bh * n_groups;
    const int32_t A = gi / ngc, Cg = gi - A * ngc;
    a = A * gh + t / gw;
    c = Cg * gw + t % gw;
    return a < G.Th[k - 1] && c < G.Tw[k - 1];
  }
  __device__ __forceinline__ QuerySet queries(int32_t item, int wave) const {
    QuerySet s;
    int32_t a, c;
    const bool ok = group_tile(item, tile_of(wave), s.bh, a, c);
    const Tile t = tile_at(G, k, ok ? a : 0, ok ? c : 0);
    s.qbase = t.base - G.C[k - 1];
    s.qnc = t.nc;
    s.qstride = t.stride;
    s.q0 = (int32_t)((wave_slab >> (4 * wave)) & 15u) * kQPerWave;
    s.q1 = ok ? t.nr * t.nc : 0;
    return s;
  }
  template <int NT>
  __device__ __forceinline__ TableCursor<KC, NT, GroupBlocks<NT>> table_cursor(int32_t item, char* lds) const {
    using L = GroupLds<NT>;
    char* glds = lds + TableLds<NT>::kBytes;
    const int T = 1 << lgT;
    const int tid = threadIdx.x;
    const GeoTable* geo = stage_geometry<NT>(G, lds);  // published by the barrier below
    if (tid < T) {
      int32_t bh, a, c;
      int32_t p = 0, n = 0;
      if (group_tile(item, tid, bh, a, c)) {
        const int32_t r = bh * G_k + a * G.Tw[k - 1] + c;
        p = row_ptr[r];
        n = row_ptr[r + 1] - p;
      }
      reinterpret_cast<int32_t*>(glds + L::kRowP)[tid] = p;
      reinterpret_cast<int32_t*>(glds + L::kRowN)[tid] = n;
    }
    __syncthreads();
    const int32_t RC = NT >> lgT;
    bool long_row = false;
    for (int t = 0; t < T; ++t) long_row |= reinterpret_cast<const int32_t*>(glds + L::kRowN)[t] > RC;
    TableCursor<KC, NT, GroupBlocks<NT>> cur;
    cur.G = geo;
    cur.blocks.col = col_idx;
    cur.blocks.nb = G.NB[k];
    cur.blocks.T = T;
    cur.blocks.lgT = lgT;
    cur.blocks.by_tile = long_row;
    cur.blocks.started = false;
    cur.blocks.seg_t = 0;
    cur.blocks.seg_off = 0;
    cur.blocks.lds = glds;
    cur.nb = G.NB[k];
    const int32_t g = kTableCap / (max_chunks_per_block > 0 ? max_chunks_per_block : 1);
    cur.group = g < NT ? (g > 0 ? g : 1) : NT;
    cur.pos = 0;
    cur.end = 0;
    cur.tn = 0;
    cur.ti = 0;
    cur.lds = lds;
    return cur;
  }
};


// LDS pipeline stages as separate arrays: alias analysis then sees that the
// direct HBM -> LDS copies into one stage cannot touch the stage being read,
// and the compiler does not wait for those copies before every LDS read.
#define SV_STAGE_ARRAYS(NSX, BYTES)                                              \
  __shared__ __attribute__((aligned(16))) char sv_stage0[BYTES];                 \
  __shared__ __attribute__((aligned(16))) char sv_stage1[BYTES];                 \
  __shared__ __attribute__((aligned(16))) char sv_stage2[(NSX) > 2 ? (BYTES) : 16]; \
  __shared__ __attribute__((aligned(16))) char sv_stage3[(NSX) > 3 ? (BYTES) : 16];

template <int S>
__device__ __forceinline__ char* stage_ptr(char* s0, char* s1, char* s2, char* s3) {
  if constexpr (S == 0) return s0;
  else if constexpr (S == 1) return s1;
  else if constexpr (S == 2) return s2;
  else return s3;
}

// Sources with a kRuns member walk listed 1-D key blocks (BlockRowSrc).
template <class Src, class = void>
constexpr bool kRunsOf = false;
template <class Src>
constexpr bool kRunsOf<Src, std::void_t<decltype(Src::kRuns)>> = Src::kRuns;
// Sources with a kRemap member map a launch position to a work item (GroupSrc).
template <class Src, class = void>
constexpr bool kRemapOf = false;
template <class Src>
constexpr bool kRemapOf<Src, std::void_t<decltype(Src::kRemap)>> = Src::kRemap;

// Running maximum before the first key: finite, so that keys that all score -inf
// leave zero weights (exp2(-inf - m) = 0) and not exp2(-inf + inf). A part of a key
// walk starts anywhere in the row, so its first keys may well be such keys.
constexpr float kNoMax = -3.402823466e38f;

// Merge of KS key splits of one workgroup (QW query waves each): the softmax maximum
// m_g and sum l_g over the splits, and in out the unnormalised sums of the accumulator
// registers [split R, (split + 1) R) (16 per 32-channel group, R = D / 2 / KS) that
// this wave finishes, added in split order. The other splits hand theirs over through the stage
// arrays s0 of SB and s1 of SB1 bytes, which every wave has finished with by the first barrier.
template <int D, int QW, int KS, int SB, int SB1 = SB>
__device__ __forceinline__ void merge_key_splits(const f32x16 (&acc)[D / 32], float m_run, float l_run, int split,
                                                 int qwave, int lane, char* s0, char* s1,
                                                 float (&ml)[KS][QW * kQPerWave][2], float& m_g, float& l_g,
                                                 float (&out)[D / 2 / KS]) {
  constexpr int R = D / 2 / KS;
  constexpr int kPart = R * 64;  // floats one wave hands to one other split
  constexpr int kHalf = SB / (kPart * 4);
  static_assert(R % 4 == 0, "output channels must split into groups of four");
  static_assert(KS * (KS - 1) * QW <= kHalf + SB1 / (kPart * 4), "split outputs must fit the stages they merge through");
  const int slot = qwave * kQPerWave + (lane & 31);
  const float l_tot = sum_halves(l_run);
  if (lane < 32) {
    ml[split][slot][0] = m_run;
    ml[split][slot][1] = l_tot;
  }
  __syncthreads();
  m_g = kNoMax;
#pragma unroll
  for (int s = 0; s < KS; ++s) m_g = fmaxf(m_g, ml[s][slot][0]);
  l_g = 0.f;
#pragma unroll
  for (int s = 0; s < KS; ++s) l_g += ml[s][slot][1] * __builtin_amdgcn_exp2f(ml[s][slot][0] - m_g);
  const float own = __builtin_amdgcn_exp2f(m_run - m_g);
  auto part = [&](int t, int from) {
    const int i = (t * (KS - 1) + (from < t ? from : from - 1)) * QW + qwave;
    char* base = i < kHalf ? s0 + i * (kPart * 4) : s1 + (i - kHalf) * (kPart * 4);
    return reinterpret_cast<float*>(base) + lane;
  };
#pragma unroll
  for (int t = 0; t < KS; ++t) {
    if (t == split) continue;
    float* to = part(t, split);
#pragma unroll
    for (int i = 0; i < R; ++i) to[i * 64] = acc[(t * R + i) / 16][(t * R + i) % 16] * own;
  }
  __syncthreads();
#pragma unroll
  for (int t = 0; t < KS; ++t) {
    if (t != split) continue;  // (a compare per split, so that register indices stay constant)
#pragma unroll
    for (int i = 0; i < R; ++i) {
      float r = 0.f;
#pragma unroll
      for (int u = 0; u < KS; ++u) r += u == t ? acc[(t * R + i) / 16][(t * R + i) % 16] * own : part(t, u)[i * 64];
      out[i] = r;
    }
  }
}

// Channel of the first of the four accumulator registers 4 i .. 4 i + 3.
__device__ __forceinline__ int channel_of(int i, int half) { return 32 * (i >> 2) + 8 * (i & 3) + 4 * half; }

// Waves (32 queries each) for a tile of that many queries.
inline int waves_for(int32_t queries) {
  if (queries <= 32) return 1;
  if (queries <= 64) return 2;
  if (queries <= 128) return 4;
  return 8;
}

// Largest chunk count of any block of scales 1..k (full and edge tiles) at kc keys per chunk.
inline int32_t max_chunks_per_block(const GeoTable& G, int k, int kc) {
  int32_t maxc = 1;
  for (int l = 1; l <= k; ++l) {
    const int32_t eh = G.eh[l - 1], ew = G.ew[l - 1];
    const int32_t rh[2] = {eh, G.h[l - 1] - (G.Th[l - 1] - 1) * eh};
    const int32_t rw[2] = {ew, G.w[l - 1] - (G.Tw[l - 1] - 1) * ew};
    for (int i = 0; i < 2; ++i)
      for (int j = 0; j < 2; ++j) {
        const int32_t nr = rh[i], nc = rw[j];
        int32_t c;
        if (nr == 1 || nc == G.w[l - 1]) c = (nr * nc + kc - 1) / kc;
        else if (nc <= kc) c = (nr + kc / nc - 1) / (kc / nc);
        else c = nr * ((nc + kc - 1) / kc);
        maxc = c > maxc ? c : maxc;
      }
  }
  return maxc;
}

}  // namespace sparvar
