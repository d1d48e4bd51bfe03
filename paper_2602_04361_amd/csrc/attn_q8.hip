// Attention over an 8-bit cache: dense, and block-sparse over CSR rows.
//
// The walk is that of the bf16 kernels (attention.hip): S^T = K Q^T, softmax in the exp2
// domain with a running maximum, O^T += V^T P^T, on 32x32x16 bf16 MFMA with K and V chunks
// staged in LDS. Codes become bf16 on their way to LDS, once a workgroup: e4m3 has 4
// significant bits and scales are powers of two, so code * 2^e is exact in bf16 and the
// conversion (one instruction for two values, the scale its operand) rounds nothing. The
// products are then those of a 16-bit cache holding the same values.
//
// A step of the pipeline: chunk i sits in one LDS stage while chunk i + 1, loaded to
// registers a step ago, is converted into the other and the loads of chunk i + 2 are
// issued; one barrier a chunk. A lane loads 16 codes (of one token, so one scale) at a time.
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
  int32_t group;    // query heads a key head
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

template <int KC>
struct SparseQ8Src : SparseSrc<KC> {
  int32_t group;
  __device__ __forceinline__ int32_t part_of(int32_t) const { return 0; }
  __device__ __forceinline__ int32_t kv_plane(const QuerySet& s) const { return s.bh / group; }
  __device__ __forceinline__ void place(const QuerySet& s, int32_t i, int32_t& plane, int32_t& row) const {
    plane = s.bh;
    row = s.qbase + (i / s.qnc) * s.qstride + i % s.qnc;
  }
};

template <int D, int NW, int KC, class Src>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(2))) void attn_q8_kernel(Q8IO io, Src src) {
  constexpr int NT = NW * 64;
  constexpr int U = D / 8;                    // 16-byte units of a bf16 row in LDS
  constexpr int kRow = D * 2;
  constexpr int kTile = KC * kRow;            // K (or V) of a chunk in LDS
  constexpr int kPieces = KC * D / 16;        // 16-code pieces of K (or V) of a chunk
  constexpr int kLoads = 2 * kPieces / NT;    // pieces a lane converts
  static_assert(2 * kPieces % NT == 0 && kPieces % 64 == 0, "pieces must split evenly, K and V by whole waves");
  __shared__ __attribute__((aligned(16))) char stage0[2 * kTile];
  __shared__ __attribute__((aligned(16))) char stage1[2 * kTile];
  __shared__ __attribute__((aligned(16))) char tsmem[Src::template table_bytes<NT>()];

  const int32_t item = swizzled_item(blockIdx.x, gridDim.x, io.swizzle);
  if (item >= io.n_items) return;
  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, half = lane >> 5;

  const QuerySet qs = src.queries(item, wave);
  const int32_t qslot = qs.q0 + l32;
  const bool qvalid = qslot < qs.q1;
  int32_t plane, qrow;
  src.place(qs, qvalid ? qslot : 0, plane, qrow);
  QFragBF16<D> qf;
  qf.load(io.q + (int64_t)plane * io.q_bh_stride + (int64_t)qrow * D, half);

  const int32_t kvp = src.kv_plane(qs);
  const uint8_t* planes[2] = {io.c.k + (int64_t)kvp * io.c.bh_stride, io.c.v + (int64_t)kvp * io.c.bh_stride};
  const uint8_t* scales[2] = {io.c.ks + (int64_t)kvp * io.c.sc_stride, io.c.vs + (int64_t)kvp * io.c.sc_stride};

  f32x16 acc[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) acc[i] = zero16();
  float m_run = kNoMax, l_run = 0.f;

  FragOffsets<D, KC> fo;
  fo.init(l32, half, lane);

  // Piece j of a lane: 16 codes of one key of K (piece below kPieces) or V. Its two units
  // of bf16 go to LDS in an order that differs between the halves of eight lanes, so that
  // eight lanes of a write meet eight different groups of banks.
  int key_of_piece[kLoads], lds_of_piece[kLoads][2];
  uint32_t off_of_piece[kLoads];
#pragma unroll
  for (int j = 0; j < kLoads; ++j) {
    const int x = (j * NT + tid) % kPieces;
    const int r = x / (D / 16), c = x % (D / 16), swap = (lane >> 2) & 1;
    key_of_piece[j] = r;
    off_of_piece[j] = 16 * c;
    const int base = ((j * NT + wave * 64) >= kPieces ? kTile : 0) + r * kRow, sw = unit_swizzle(r) & (U - 1);
    lds_of_piece[j][0] = base + 16 * ((2 * c + swap) ^ sw);
    lds_of_piece[j][1] = base + 16 * ((2 * c + 1 - swap) ^ sw);
  }
  const bool swapped = (lane >> 2) & 1;

  u32x4 raw[kLoads];
  uint32_t raw_s[kLoads];
  auto load = [&](const Chunk& c) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int is_v = (j * NT + wave * 64) >= kPieces;
      const uint32_t tok = (uint32_t)chunk_token(c, chunk_slot(key_of_piece[j], c.count));
      raw[j] = *reinterpret_cast<const u32x4*>(planes[is_v] + (tok * D + off_of_piece[j]));
      raw_s[j] = scales[is_v][tok >> io.c.lg];
    }
  };
  auto convert = [&](char* st) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const float f = scale_of_byte(raw_s[j]);
      u32x4 a, b;
      uint32_t w[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) decode4_bf16(raw[j][i], f, w[2 * i], w[2 * i + 1]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        a[i] = swapped ? w[4 + i] : w[i];
        b[i] = swapped ? w[i] : w[4 + i];
      }
      *reinterpret_cast<u32x4*>(st + lds_of_piece[j][0]) = a;
      *reinterpret_cast<u32x4*>(st + lds_of_piece[j][1]) = b;
    }
  };

  auto compute = [&](const char* kst, int32_t count) {
    f32x16 st[KC / 32];
    qk_chunk<D, KC>(kst, fo, qf, st);
    if (count < KC) mask_tail<KC>(st, count, half);
    const float mx = row_max<KC>(st, io.scale_log2);
    if (__builtin_amdgcn_ballot_w64(mx > m_run + 8.f)) {
      const float m_new = fmaxf(m_run, mx);
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      l_run *= alpha;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) acc[i] *= alpha;
      m_run = m_new;
    }
    bf16x8 pf[KC / 16];
    l_run += exp_pack<KC>(st, io.scale_log2, m_run, pf);
    pv_chunk<D, KC>(kst, fo, pf, acc);
  };

  auto cur = [&]() {
    if constexpr (Src::kSparse) return src.template table_cursor<NT>(item, tsmem);
    else return src.cursor(item, qs);
  }();
  // One pass over what the cursor holds (a block table is filled again between passes,
  // with a barrier, so both stages are free when a pass starts).
  auto walk = [&]() {
    Chunk c0, c1;
    if (!cur.next(c0)) return;
    load(c0);
    convert(stage0);
    bool more = cur.next(c1);
    if (more) load(c1);
    auto step = [&](char* now, char* then) -> bool {
      __syncthreads();
      const int32_t count = c0.count;
      const bool go_on = more;
      if (more) {
        convert(then);
        c0 = c1;
        more = cur.next(c1);
        if (more) load(c1);
      }
      compute(now, count);
      return go_on;
    };
    for (;;) {
      if (!step(stage0, stage1)) break;
      if (!step(stage1, stage0)) break;
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

  const float l_tot = sum_halves(l_run);
  if (!qvalid) return;
  const int64_t orow = (int64_t)plane * io.o_rows + qrow;
  if (io.part_o) {
    const int64_t prow = (int64_t)src.part_of(item) * io.rows + orow;
    float* op = io.part_o + prow * D;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<float4*>(op + 32 * dt + 8 * j + 4 * half) =
            make_float4(acc[dt][4 * j], acc[dt][4 * j + 1], acc[dt][4 * j + 2], acc[dt][4 * j + 3]);
    if (half == 0) io.part_ml[prow] = make_float2(m_run, l_tot);
    return;
  }
  const float inv = l_tot > 0.f ? 1.f / l_tot : 0.f;
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
  if (io.lse && half == 0) io.lse[orow] = l_tot > 0.f ? (m_run + __builtin_log2f(l_tot)) * kLn2 : -INFINITY;
}

// Joins the parts of every row, in order: a thread takes four channels of a row. A part
// without keys has no sum and its values are not read.
template <int D>
__global__ __launch_bounds__(256) void join_parts_kernel(Q8IO io, int32_t parts) {
  const int32_t row = blockIdx.x * (1024 / D) + threadIdx.x / (D / 4);
  const int c = threadIdx.x % (D / 4) * 4;
  if (row >= io.rows) return;
  float m = kNoMax;
  for (int p = 0; p < parts; ++p) m = fmaxf(m, io.part_ml[(int64_t)p * io.rows + row].x);
  float l = 0.f, r[4] = {0.f, 0.f, 0.f, 0.f};
  for (int p = 0; p < parts; ++p) {
    const int64_t prow = (int64_t)p * io.rows + row;
    const float2 ml = io.part_ml[prow];
    if (!(ml.y > 0.f)) continue;
    const float f = __builtin_amdgcn_exp2f(ml.x - m);
    const float4 a = *reinterpret_cast<const float4*>(io.part_o + prow * D + c);
    l += ml.y * f;
    r[0] += a.x * f;
    r[1] += a.y * f;
    r[2] += a.z * f;
    r[3] += a.w * f;
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  uint2 w;
  w.x = pack_bf16x2(r[0] * inv, r[1] * inv);
  w.y = pack_bf16x2(r[2] * inv, r[3] * inv);
  *reinterpret_cast<uint2*>(io.o + (int64_t)row * D + c) = w;
  if (io.lse && c == 0) io.lse[row] = l > 0.f ? (m + __builtin_log2f(l)) * kLn2 : -INFINITY;
}

// Waves, slabs and parts of a dense call.
struct DenseQ8Plan {
  int waves;
  int32_t slabs, parts;
};

DenseQ8Plan dense_plan(int32_t planes, int32_t group, int32_t n_q, int32_t n_kv, int num_cu) {
  DenseQ8Plan p;
  const int64_t rows = (int64_t)group * n_q;
  p.waves = rows <= 32 ? 1 : rows <= 64 ? 2 : 4;
  p.slabs = (int32_t)((rows + 32 * p.waves - 1) / (32 * p.waves));
  // Parts: as many as fill two workgroups a CU, of at least four chunks each.
  const int64_t items = planes * (int64_t)p.slabs, want = (2 * (int64_t)num_cu + items - 1) / items;
  const int64_t most = (n_kv + 255) / 256;
  p.parts = (int32_t)(want < most ? want : most);
  if (p.parts > 64) p.parts = 64;
  return p;
}

template <int D, int NW, int KC, class Src>
hipError_t launch_one(Q8IO io, const Src& src, hipStream_t stream) {
  int32_t grid = io.n_items;
  if (io.swizzle) grid = (grid + 7) / 8 * 8;
  hipLaunchKernelGGL((attn_q8_kernel<D, NW, KC, Src>), dim3(grid), dim3(NW * 64), 0, stream, io, src);
  return hipGetLastError();
}

int64_t part_floats(int32_t parts, int64_t rows, int32_t d) { return (int64_t)parts * rows * (d + 2); }

}  // namespace

int64_t dense_q8_workspace(int32_t B, int32_t H, int32_t H_kv, int32_t n_q, int32_t n_kv, int32_t d, int num_cu) {
  const DenseQ8Plan p = dense_plan(B * H_kv, H / H_kv, n_q, n_kv, num_cu);
  return p.parts > 1 ? 4 * part_floats(p.parts, (int64_t)B * H * n_q, d) : 0;
}

hipError_t launch_dense_attn_q8(const DenseQ8Args& a, hipStream_t stream) {
  const int32_t group = a.H / a.H_kv;
  DenseQ8Plan p = dense_plan(a.B * a.H_kv, group, a.n_q, a.n_kv, a.num_cu);
  if (!a.workspace) p.parts = 1;
  Q8IO io;
  io.q = static_cast<const bf16_bits*>(a.q);
  io.o = static_cast<bf16_bits*>(a.o);
  io.lse = a.lse;
  io.q_bh_stride = a.q_bh_stride;
  io.c = a.c8;
  io.o_rows = a.n_q;
  io.n_items = a.B * a.H_kv * p.slabs * p.parts;
  io.swizzle = a.swizzle;
  io.group = group;
  io.scale_log2 = a.softmax_scale * kLog2e;
  io.rows = a.B * a.H * a.n_q;
  io.part_o = p.parts > 1 ? a.workspace : nullptr;
  io.part_ml = p.parts > 1 ? reinterpret_cast<float2*>(a.workspace + (int64_t)p.parts * io.rows * a.d) : nullptr;
  DenseQ8Src<64> src;
  src.n_q = a.n_q;
  src.n_kv = a.n_kv;
  src.H_kv = a.H_kv;
  src.group = group;
  src.slabs = p.slabs;
  src.q_per_wg = 32 * p.waves;
  src.parts = p.parts;
  src.kv_len = a.kv_len;
  hipError_t e = hipErrorInvalidValue;
#define SV_DENSE(DD, NN) \
  if (a.d == DD && p.waves == NN) e = launch_one<DD, NN, 64>(io, src, stream);
  SV_DENSE(64, 1) SV_DENSE(64, 2) SV_DENSE(64, 4) SV_DENSE(128, 1) SV_DENSE(128, 2) SV_DENSE(128, 4)
#undef SV_DENSE
  if (e != hipSuccess || p.parts == 1) return e;
  const int per = 1024 / a.d;
  const int32_t grid = (io.rows + per - 1) / per;
  if (a.d == 128) hipLaunchKernelGGL((join_parts_kernel<128>), dim3(grid), dim3(256), 0, stream, io, p.parts);
  else hipLaunchKernelGGL((join_parts_kernel<64>), dim3(grid), dim3(256), 0, stream, io, p.parts);
  return hipGetLastError();
}

hipError_t launch_sparse_attn_q8(const SparseQ8Args& a, hipStream_t stream) {
  const GeoTable& G = *a.G;
  const int32_t tile_q = G.eh[a.k - 1] * G.ew[a.k - 1], G_k = tiles_of(G, a.k);
  const int nw = waves_for(tile_q);
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
  io.group = a.H / a.H_kv;
  io.scale_log2 = a.softmax_scale * kLog2e;
  io.part_o = nullptr;
  io.part_ml = nullptr;
  io.rows = a.BH * io.o_rows;
  SparseQ8Src<64> src;
  src.group = io.group;
  src.max_chunks_per_block = max_chunks_per_block(G, a.k, 64);
  src.G = G;
  src.row_ptr = a.row_ptr;
  src.col_idx = a.col_idx;
  src.schedule = a.schedule;
  src.k = a.k;
  src.G_k = G_k;
  src.q_per_wg = qpw;
  src.slabs = slabs;
  src.n_rows = a.BH * G_k;
#define SV_SPARSE(DD, NN) \
  if (a.d == DD && nw == NN) return launch_one<DD, NN, 64>(io, src, stream);
  SV_SPARSE(64, 1) SV_SPARSE(64, 2) SV_SPARSE(64, 4) SV_SPARSE(64, 8)
  SV_SPARSE(128, 1) SV_SPARSE(128, 2) SV_SPARSE(128, 4) SV_SPARSE(128, 8)
#undef SV_SPARSE
  return hipErrorInvalidValue;
}

}  // namespace sparvar
