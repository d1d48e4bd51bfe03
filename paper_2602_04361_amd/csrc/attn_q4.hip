// Attention over a 4-bit cache: dense, and block-sparse over CSR rows.
//
// The walk is that of the kernels over an 8-bit cache (attn_q8.hip): S^T = K Q^T, softmax in the
// exp2 domain with a running maximum, O^T += V^T P^T. K = c 2^e with a scale byte a key and 32
// channels is what the 32x32x64 product of 4-bit codes takes: a lane holds the 32 channels of one
// key and half, and the byte that goes with them. So K goes from memory through LDS to the matrix
// cores as it is, beside Q as the sum of two e4m3 values (QFragF8), at the rate of one bf16 product.
// V becomes bf16 on its way to LDS, once a workgroup: c 2^e has 2 significant bits, so the
// conversion (one instruction for two values, the scale its operand) rounds nothing. A lane's
// codes of V belong to one scale.
//
// Scores, maxima, sums and O are held in 32 bits. The probabilities are rounded to bf16 for the
// product with V, each off by at most 2^-8 of itself, as in the bf16 kernels (the sum that
// divides them is that of the 32-bit ones).
//
// Many rows are bound by the matrix units (busy 48% of the time in the case below) and the exponentials
// and packing in between (vector units 43%), which hardly overlap, and by the power that both draw: 2 x 16 heads,
// 4096 x 10521, d = 128, with LSE 581 to 639 us by card (1.22 to 1.11 PFLOP/s; one large bf16 product runs at 1.34),
// the 8-bit cache on the same cards 571 to 600. Block-sparse, the same heads' 64 x 64 scale with 1355 tokens
// a row: 124 to 127 us, bound the same way at 37% and 48%, with every second wave's worth of V
// converted for 64 rows alone. Short rows are bound by what stands before the first product (some 8 us). In turn on one
// card, rows of 14 chosen blocks: 130.5 us and 131.7 over 8 bits, 48 x 36 at d = 64 27.7 and 28.7, dense 591 and 586.
#include "attn_codes.h"
#include "q4.h"
#include "q8.h"

namespace sparvar {

namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;

struct Q4IO : RowsIO {
  Q4View c;
};

// Which codes of a wave's 16 rows of V a lane loads and converts: four lanes take a row, 32 codes
// each (16 at D = 64). Eight neighbouring lanes, whose 16-byte writes go out together, take a row and
// the one four further, which the swizzle puts in the other of two neighbouring units. At D = 128 that
// leaves two lanes to a group of banks (14% of the LDS cycles of a dense call); without that, by other
// rows in a lane's neighbours or by units written in another order, the dense call took as long and the
// block-sparse one above 127 us against 124.
__device__ __forceinline__ void lane_quarter(int lane, int& row, int& col) {
  row = ((lane >> 3) & 3) + ((lane >> 2) & 1) * 4 + (lane >> 5) * 8;
  col = lane & 3;
}

// A lane's codes of V, and their scale.
template <int D>
struct VPiece {
  uint32_t w[D / 32];
  uint32_t byte;
  __device__ __forceinline__ void load(const uint8_t* v, const uint8_t* vs, uint32_t tok, int col) {
    const uint8_t* p = v + (tok * (D / 2) + col * (D / 8));
    if constexpr (D == 128) {
      const u32x4 r = *reinterpret_cast<const u32x4*>(p);
      w[0] = r[0], w[1] = r[1], w[2] = r[2], w[3] = r[3];
    } else {
      const uint2 r = *reinterpret_cast<const uint2*>(p);
      w[0] = r.x, w[1] = r.y;
    }
    byte = vs[tok * (D / 32) + (D == 128 ? col : col >> 1)];
  }
  // Unit x of the piece goes to `row` at its place among the swizzled units.
  __device__ __forceinline__ void put(char* row, int col, int sw) const {
    const float f = q4_scale(byte);
#pragma unroll
    for (int x = 0; x < D / 32; ++x)
      *reinterpret_cast<u32x4*>(row + 16 * (((D / 32) * col + x) ^ sw)) = q4_decode8_bf16(w[x], f);
  }
};

// Scale bytes of a key, those of the lane's half in byte 0 and (D = 128) byte 2.
template <int D>
__device__ __forceinline__ uint32_t key_scales(const uint8_t* ks, uint32_t tok, int half) {
  if constexpr (D == 128) return *reinterpret_cast<const uint32_t*>(ks + tok * 4) >> (8 * half);
  else return (uint32_t)ks[tok * 2 + half];
}

// c += K Q^T over 64 channels: a the codes of 32 keys, ks their scales, of which step t takes byte
// 2 t. Of the queries' scale, byte 0 goes with hi and byte 1 with lo.
template <int D, int T>
__device__ __forceinline__ f32x16 mfma_k4(u32x4 a, uint32_t ks, const QFragF8<D, true>& q, f32x16 c) {
#if defined(__HIP_DEVICE_COMPILE__)
  const i32x8 k = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
  c = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k, q.hi[T], c, 4, 0, 2 * T, (int)ks, 0, q.scale);
  c = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k, q.lo[T], c, 4, 0, 2 * T, (int)ks, 1, q.scale);
#endif
  return c;
}

// K codes in LDS: rows of D / 2 bytes, 16-byte unit u of row r at u ^ key_swizzle(r): four or eight
// rows fill the 256 bytes of the banks.
template <int D>
__device__ __forceinline__ int key_swizzle(int r) {
  return D == 128 ? (r >> 2) & 3 : (r >> 3) & 1;
}

// QW waves of 32 queries walk the keys in chunks of 64, or (KS > 1) KS such sets, each a part of
// them with LDS of its own, joined through it at the end. While a chunk is computed, the next one's K
// is copied to the other K tile and its V loaded to registers, to be converted into the one V tile
// between two barriers.
template <int D, int QW, int KS, class Src>
__global__ __launch_bounds__(QW * KS * 64) __attribute__((amdgpu_waves_per_eu(2))) void attn_q4_kernel(Q4IO io, Src src) {
  constexpr int KC = 64, NT = QW * KS * 64;
  constexpr int kRow = D * 2;                 // bytes of a V row in LDS
  constexpr int kKRow = D / 2;                // of a K row
  constexpr int kKTile = KC * kKRow, kVTile = KC * kRow;
  constexpr int U4 = D / 32;                  // 16-byte units of a K row
  // V rows go to waves 16 at a time, K units 64 at a time; where there are more waves than V
  // rows, the second half of them copies K.
  constexpr bool kHalf = QW * 16 > KC;
  constexpr int kVSteps = kHalf ? 1 : KC / (QW * 16);
  constexpr int kKCopies = KC * U4 / 64;      // a wave's worth each
  constexpr int kKWaves = kHalf ? QW / 2 : QW;
  constexpr int kKSteps = kKCopies > kKWaves ? kKCopies / kKWaves : 1;
  static_assert(kHalf ? QW * 16 == 2 * KC : KC % (QW * 16) == 0, "V rows must split evenly");
  static_assert(kKCopies % kKSteps == 0, "K units must split evenly");
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
  auto cur = [&]() {
    if constexpr (Src::kSparse) return src.template packed_cursor<NT>(item, tsmem);
    else return src.cursor(item, qs);
  }();
  int32_t entry = 0;
  if constexpr (Src::kSparse) entry = cur.entry();
  QFragF8<D, true> qf;
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

  // K fragments: unit 2 t + half of row l32 (rows 32 apart share their swizzle)
  int k_off[D / 64];
#pragma unroll
  for (int t = 0; t < D / 64; ++t) k_off[t] = l32 * kKRow + 16 * ((2 * t + half) ^ key_swizzle<D>(l32));
  VOffsets<D, KC> vo;
  vo.init(l32, half, lane);

  // V: a lane's piece of row vrow, and of rows QW * 16 further (a multiple of 16, so LDS offsets
  // differ by a constant)
  char* const vtile = vtiles[split];
  int vrow, vcol;
  lane_quarter(lane, vrow, vcol);
  vrow += wave * 16;
  const int kwave = kHalf ? wave - QW / 2 : wave;
  const bool does_v = !kHalf || wave < QW / 2, does_k = kwave >= 0 && kwave < kKCopies / kKSteps;  // wave-uniform
  char* const v_lds = vtile + vrow * kRow;
  const int v_sw = unit_swizzle(vrow) & (D / 8 - 1);
  // K: a direct copy of the wave covers 64 units in a row; a lane fetches the unit that the
  // swizzle puts at its place
  const int k_first = kwave * kKSteps * 64;
  const int k_row = (k_first + lane) / U4, k_unit = (k_first + lane) % U4;

  VPiece<D> raw[kVSteps];
  uint32_t k_scale[KC / 32], k_scale_next[KC / 32];
  auto load = [&](const auto& c, char* kdst) {
    if (does_k) {
      const int32_t base = slot_base(c, k_row);
#pragma unroll
      for (int j = 0; j < kKSteps; ++j) {
        const int r = k_row + j * (64 / U4);
        const uint32_t tok = token_at(c, base, j * (64 / U4));
        dma16(kp + (tok * kKRow + 16 * (k_unit ^ key_swizzle<D>(r))), kdst + (k_first + j * 64) * 16);
      }
    }
    if (does_v) {
      const int32_t base = slot_base(c, vrow);
#pragma unroll
      for (int j = 0; j < kVSteps; ++j) raw[j].load(vp, vsp, token_at(c, base, j * QW * 16), vcol);
    }
    if constexpr (Src::kSparse) {  // (the tokens of slots l32 and 32 + l32)
      const auto t = __builtin_amdgcn_permlane32_swap(c.tok, c.tok, false, false);
      k_scale_next[0] = key_scales<D>(ksp, (uint32_t)t[0], half);
      k_scale_next[1] = key_scales<D>(ksp, (uint32_t)t[1], half);
    } else {
#pragma unroll
      for (int kt = 0; kt < KC / 32; ++kt) k_scale_next[kt] = key_scales<D>(ksp, token_at(c, l32, 32 * kt), half);
    }
  };
  // The chunk loaded last becomes the one to be computed: V to LDS, K's copies arrived.
  auto take = [&]() {
    if (does_v) {
#pragma unroll
      for (int j = 0; j < kVSteps; ++j) raw[j].put(v_lds + j * (QW * 16 * kRow), vcol, v_sw);
    }
#pragma unroll
    for (int kt = 0; kt < KC / 32; ++kt) k_scale[kt] = k_scale_next[kt];
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
  };

  // One chunk, K in kt_, V in vtile; `next` issues the loads of the next one. The order of the
  // LDS reads is pinned: K first, V under the products of S.
  auto compute = [&](const char* kt_, int32_t count, auto next) {
    f32x16 st[KC / 32];
    u32x4 kf[KC / 32][D / 64];
    bf16x8 vf[KC / 16][D / 32], pf[KC / 16];
#pragma unroll
    for (int kt = 0; kt < KC / 32; ++kt)
#pragma unroll
      for (int t = 0; t < D / 64; ++t) kf[kt][t] = *reinterpret_cast<const u32x4*>(kt_ + k_off[t] + kt * 32 * kKRow);
    __builtin_amdgcn_sched_barrier(0);
    next();
    __builtin_amdgcn_sched_barrier(0);
    constexpr int kProducts = KC / 32 * (D / 64), kV = KC / 16 * (D / 32);  // V fragments to read under them
#pragma unroll
    for (int kt = 0; kt < KC / 32; ++kt) st[kt] = zero16();
#pragma unroll
    for (int i = 0; i < kProducts; ++i) {
      const int kt = i / (D / 64), t = i % (D / 64);
      if (t == 0) st[kt] = mfma_k4<D, 0>(kf[kt][0], k_scale[kt], qf, st[kt]);
      if constexpr (D == 128) {
        if (t == 1) st[kt] = mfma_k4<D, 1>(kf[kt][1], k_scale[kt], qf, st[kt]);
      }
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
    while (cur.fill(entry)) {
      walk();
      if (!cur.more()) break;
      entry = cur.entry();
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
// chunk's codes in flight. K goes from registers to the products, converted: a lane holds half of a
// key's channels, and as a sum over channels may run in any order, step s takes channels 8 s .. of
// each half. V goes through a piece of LDS of the wave's own, for the transposing read. The four
// waves of a workgroup take every fourth chunk of a part and join at the end. (2 x 16 heads, 256 x 521, d = 128:
// 9.9 us; 1 x 8, 1024 x 2521: 20.)
constexpr int kRowWaves = 4;

template <int D>
__global__ __launch_bounds__(kRowWaves * 64) __attribute__((amdgpu_waves_per_eu(2)))
void attn_q4_rows_kernel(Q4IO io, DenseRowsSrc<32> src) {
  constexpr int KC = 32, kRow = D * 2;
  constexpr int kK = D / 64;             // 16-byte pieces of a lane's half of a key
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
  lane_quarter(lane, vrow, vcol);
  const int sw = unit_swizzle(vrow) & (D / 8 - 1);

  u32x4 kr[kK];
  VPiece<D> vr[2];
  uint32_t ksc;  // scale bytes of the lane's half of its key
  const DenseCursor<KC> cur = src.cursor(item, qs);
  auto load = [&](int32_t pos) {
    const int32_t last = cur.n - 1;
    const uint32_t kt = (uint32_t)(pos + l32 < last ? pos + l32 : last);
#pragma unroll
    for (int i = 0; i < kK; ++i) kr[i] = *reinterpret_cast<const u32x4*>(kp + (kt * (D / 2) + half * (D / 4) + 16 * i));
    if constexpr (D == 128) ksc = *reinterpret_cast<const uint16_t*>(ks + (kt * 4 + 2 * half));
    else ksc = ks[kt * 2 + half];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int32_t r = pos + vrow + 16 * j;
      vr[j].load(vp, vs, (uint32_t)(r < last ? r : last), vcol);
    }
  };
  int32_t pos = cur.pos + wave * KC;
  if (pos < cur.n) load(pos);
  while (pos < cur.n) {
    // V to LDS, K to the products
#pragma unroll
    for (int j = 0; j < 2; ++j) vr[j].put(tile + (vrow + 16 * j) * kRow, vcol, sw);
    wave_fence();
    f32x16 st[1] = {zero16()};
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      const float f = q4_scale((ksc >> (8 * (s / 4))) & 0xff);
      st[0] = mfma_bf16(as_bf16x8(q4_decode8_bf16(kr[s / 4][s & 3], f)), qf[s], st[0]);
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

// Up to 16 rows a workgroup: the same on 16x16x32 products, half the work of the wider ones on rows
// that are mostly not there. A lane holds a quarter of a key's channels: 16 bytes of codes of one
// scale at d = 128, and sixteen neighbouring keys' are 1 KB in a row for a load of the wave. Bound by
// memory: one token of 4 x 32 heads on 8, up to 42521 keys (150 MB) 32 us and 4.7 for the join of 16 parts, where a
// large copy of as much takes 29.
__device__ __forceinline__ f32x4 mfma16_bf16(bf16x8 a, bf16x8 b, f32x4 c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
#else
  return c;
#endif
}

// x of the lanes 16 apart and 32 apart, joined.
__device__ __forceinline__ HalfPair rows16(float x) {
#if defined(__HIP_DEVICE_COMPILE__)
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return HalfPair{__uint_as_float(r[0]), __uint_as_float(r[1])};
#else
  return HalfPair{x, x};
#endif
}
__device__ __forceinline__ float max_quarters(float x) {
  const HalfPair p = rows16(x);
  return max_halves(fmaxf(p.lo, p.hi));
}
__device__ __forceinline__ float sum_quarters(float x) {
  const HalfPair p = rows16(x);
  return sum_halves(p.lo + p.hi);
}

template <int D>
__global__ __launch_bounds__(kRowWaves * 64) __attribute__((amdgpu_waves_per_eu(3)))
void attn_q4_few_kernel(Q4IO io, DenseRowsSrc<32> src) {
  constexpr int KC = 32, kRow = D * 2, kTile = KC * kRow;
  constexpr int kC = D / 16;   // tiles of 16 channels
  constexpr int kDeep = 2;     // chunks in flight
  __shared__ __attribute__((aligned(16))) char tiles[kRowWaves][kTile];
  __shared__ float2 ml[kRowWaves][16];

  const int32_t item = swizzled_item(blockIdx.x, gridDim.x, io.swizzle);
  if (item >= io.n_items) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, quarter = lane >> 4;

  const QuerySet qs = src.queries(item, 0);
  const uint8_t* kp = io.c.k + (int64_t)qs.bh * io.c.bh_stride;
  const uint8_t* vp = io.c.v + (int64_t)qs.bh * io.c.bh_stride;
  const uint8_t* ks = io.c.ks + (int64_t)qs.bh * io.c.sc_stride;
  const uint8_t* vs = io.c.vs + (int64_t)qs.bh * io.c.sc_stride;
  int vrow, vcol;
  lane_quarter(lane, vrow, vcol);
  const int sw = unit_swizzle(vrow) & (D / 8 - 1);
  const DenseCursor<KC> cur = src.cursor(item, qs);

  VPiece<D> kr[kDeep][2], vr[kDeep][2];
  auto load = [&](int i, int32_t pos) {
    const int32_t last = cur.n - 1;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int32_t k = pos + l16 + 16 * j, v = pos + vrow + 16 * j;
      kr[i][j].load(kp, ks, (uint32_t)(k < last ? k : last), quarter);
      vr[i][j].load(vp, vs, (uint32_t)(v < last ? v : last), vcol);
    }
  };
  int32_t pos = cur.pos + wave * KC;
#pragma unroll
  for (int i = 0; i < kDeep; ++i)
    if (pos + i * kRowWaves * KC < cur.n) load(i, pos + i * kRowWaves * KC);

  const bool qvalid = qs.q0 + l16 < qs.q1;
  int32_t plane, qrow;
  src.place(qs, qvalid ? qs.q0 + l16 : qs.q0, plane, qrow);
  const bf16_bits* q = io.q + (int64_t)plane * io.q_bh_stride + (int64_t)qrow * D + quarter * (D / 4);
  bf16x8 qf[D / 32];
#pragma unroll
  for (int s = 0; s < D / 32; ++s) qf[s] = as_bf16x8(ldg16(q + 8 * s));

  f32x4 acc[kC];
#pragma unroll
  for (int i = 0; i < kC; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = kNoMax, l_run = 0.f;

  // V^T: channels 16 i .. of keys 4 quarter .. + 3, and of those 16 further
  char* const tile = tiles[wave];
  const int tr_key = 4 * quarter + (l16 >> 2), tr_q = lane & 3, tr_sw = unit_swizzle(tr_key) & (D / 8 - 1);
  int v_off[kC];
#pragma unroll
  for (int i = 0; i < kC; ++i) v_off[i] = tr_key * kRow + 16 * ((2 * i + (tr_q >> 1)) ^ tr_sw) + (tr_q & 1) * 8;

  while (pos < cur.n) {
#pragma unroll
    for (int i = 0; i < kDeep; ++i) {
      if (pos >= cur.n) break;
#pragma unroll
      for (int j = 0; j < 2; ++j) vr[i][j].put(tile + (vrow + 16 * j) * kRow, vcol, sw);
      wave_fence();
      f32x4 st[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        st[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        const float f = q4_scale(kr[i][j].byte);
#pragma unroll
        for (int s = 0; s < D / 32; ++s) st[j] = mfma16_bf16(as_bf16x8(q4_decode8_bf16(kr[i][j].w[s], f)), qf[s], st[j]);
      }
      const int32_t lim = cur.n - pos - 4 * quarter;  // keys from the lane's first on
      const int32_t next = pos + kDeep * kRowWaves * KC;
      if (next < cur.n) load(i, next);
      if (cur.n - pos < KC) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (16 * j + r >= lim) st[j][r] = -INFINITY;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) mx = fmaxf(mx, st[j][r]);
      mx = max_quarters(mx) * io.scale_log2;
      if (__builtin_amdgcn_ballot_w64(mx > m_run + 8.f)) {
        const float m_new = fmaxf(m_run, mx), alpha = __builtin_amdgcn_exp2f(m_run - m_new);
        l_run *= alpha;
#pragma unroll
        for (int c = 0; c < kC; ++c) acc[c] *= alpha;
        m_run = m_new;
      }
      u32x4 pw;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float p[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[j][r], io.scale_log2, -m_run));
        l_run += (p[0] + p[1]) + (p[2] + p[3]);
        pw[2 * j] = pack_bf16x2(p[0], p[1]);
        pw[2 * j + 1] = pack_bf16x2(p[2], p[3]);
      }
#pragma unroll
      for (int c = 0; c < kC; ++c) {
        const i16x4 lo = lds_read_tr(tile + v_off[c]), hi = lds_read_tr(tile + v_off[c] + 16 * kRow);
        const uint2 a = __builtin_bit_cast(uint2, lo), b = __builtin_bit_cast(uint2, hi);
        acc[c] = mfma16_bf16(as_bf16x8(u32x4{a.x, a.y, b.x, b.y}), as_bf16x8(pw), acc[c]);
      }
      wave_fence();
      pos += kRowWaves * KC;
    }
  }

  // Join the waves: the row's maximum and sum, then each wave's registers through its tile; wave w
  // finishes a quarter of the channels, in wave order.
  const float l_own = sum_quarters(l_run);
  if (quarter == 0) ml[wave][l16] = make_float2(m_run, l_own);
  __syncthreads();
  float m_g = kNoMax, l_g = 0.f;
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) m_g = fmaxf(m_g, ml[w][l16].x);
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) l_g += ml[w][l16].y * __builtin_amdgcn_exp2f(ml[w][l16].x - m_g);
  const float own = __builtin_amdgcn_exp2f(m_run - m_g);
  const float inv = io.part_o ? 1.f : (l_g > 0.f ? 1.f / l_g : 0.f);
  const int64_t orow = (int64_t)plane * io.o_rows + qrow;
  const int64_t prow = (int64_t)src.part_of(item) * io.rows + orow;
  static_assert(kC * 4 * 256 == kTile, "a wave's sums fill its tile");
  float* to = reinterpret_cast<float*>(tile) + lane;
#pragma unroll
  for (int c = 0; c < kC; ++c)
#pragma unroll
    for (int r = 0; r < 4; ++r) to[(4 * c + r) * 64] = acc[c][r] * own;
  __syncthreads();
  if (!qvalid) return;
#pragma unroll
  for (int i = 0; i < kC / kRowWaves; ++i) {
    const int c = wave * (kC / kRowWaves) + i, ch = 16 * c + 4 * quarter;
    float r[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kRowWaves; ++w)
#pragma unroll
      for (int e = 0; e < 4; ++e) r[e] += reinterpret_cast<const float*>(tiles[w])[(4 * c + e) * 64 + lane];
    if (io.part_o) {
      *reinterpret_cast<float4*>(io.part_o + prow * D + ch) = make_float4(r[0], r[1], r[2], r[3]);
    } else {
      uint2 w;
      w.x = pack_bf16x2(r[0] * inv, r[1] * inv);
      w.y = pack_bf16x2(r[2] * inv, r[3] * inv);
      *reinterpret_cast<uint2*>(io.o + orow * D + ch) = w;
    }
  }
  if (wave == 0 && quarter == 0) {
    if (io.part_o) io.part_ml[prow] = make_float2(m_g, l_g);
    else if (io.lse) io.lse[orow] = lse_of(m_g, l_g);
  }
}

// Costs of the forms (plan_dense). Those of the wide forms are the ones over an 8-bit cache, whose walk
// is the same; those of few rows fit 40 calls of 1 to 4096 rows a head over 85 to 42521 keys, d = 64 and 128,
// every form forced: the form taken is within 5% of the best in all but two (within 14%). us at d = 128 by 16
// rows a workgroup, 32, and the best of the others: 12 heads, 160 x 600 8.5 / 9.4 / -; 16 x 4 rows on each of 4
// heads, 1200 keys 10.6 / 10.6 (in 16 parts) / -; 2 x 16 heads, 256 x 521 10.8 / 9.9 / 15.0, 576 x 1497
// 32.8 / 29.7 / 30.6, 1024 x 2521 - / 57.8 / 49.3; 8 heads, 1024 x 2521 24.0 / 20.0 / -. One token of 4 x 32 heads
// on 8, 42521 keys: 40.1 in 16 or 24 parts, 42.6 in 48.
constexpr DenseForm kDenseForms[2][6] = {
    // d = 64, d = 128
    {{0, 1, 3.f, .6f, 0.f, .20f}, {2, 4, 2.5f, 3.f, 0.f, 1.38f}, {4, 1, 3.f, 1.3f, .2f, .53f}, {4, 2, 4.5f, 4.4f, 0.f, 1.15f},
     {8, 1, 4.f, 4.4f, 0.f, 1.12f}, {0, 0, 2.f, .4f, .03f, .12f, 16}},
    {{0, 1, 2.f, 2.2f, 0.f, .32f}, {2, 4, 5.f, 4.5f, 0.f, 1.92f}, {4, 1, 3.5f, 3.f, .3f, .92f}, {4, 2, 5.5f, 6.f, 0.f, 1.8f},
     {8, 1, 5.f, 6.f, 0.f, 1.77f}, {0, 0, 2.f, .8f, .1f, .2f, 16}}};

DensePlan dense_plan(int32_t planes, int32_t group, int32_t n_q, int32_t n_kv, int32_t d, int num_cu, bool may_split) {
  return plan_dense(kDenseForms[d == 128], 1.0625f * d, planes, group, n_q, n_kv, d, num_cu, may_split);
}

template <int D, int QW, int KS, class Src>
hipError_t launch_one(const Q4IO& io, const Src& src, hipStream_t stream) {
  hipLaunchKernelGGL((attn_q4_kernel<D, QW, KS, Src>), dim3(padded_grid(io)), dim3(QW * KS * 64), 0, stream, io, src);
  return hipGetLastError();
}

}  // namespace

int64_t dense_q4_workspace(int32_t B, int32_t H, int32_t H_kv, int32_t n_q, int32_t n_kv, int32_t d, int num_cu) {
  const DensePlan p = dense_plan(B * H_kv, H / H_kv, n_q, n_kv, d, num_cu, true);
  return p.parts > 1 ? 4 * part_floats(p.parts, (int64_t)B * H * n_q, d) : 0;
}

CodesForm dense_q4_form(int32_t B, int32_t H, int32_t H_kv, int32_t n_q, int32_t n_kv, int32_t d, int num_cu, bool workspace) {
  const DensePlan p = dense_plan(B * H_kv, H / H_kv, n_q, n_kv, d, num_cu, workspace);
  return CodesForm{p.waves, p.sets, p.parts};
}

hipError_t launch_dense_attn_q4(const DenseQ4Args& a, hipStream_t stream) {
  const int32_t group = a.H / a.H_kv;
  const DensePlan p = dense_plan(a.B * a.H_kv, group, a.n_q, a.n_kv, a.d, a.num_cu, a.workspace != nullptr);
  Q4IO io;
  io.q = static_cast<const bf16_bits*>(a.q);
  io.o = static_cast<bf16_bits*>(a.o);
  io.lse = a.lse;
  io.q_bh_stride = a.q_bh_stride;
  io.c = a.c4;
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
    src.q_per_wg = p.rows;
    src.parts = p.parts;
    src.kv_len = a.kv_len;
    return src;
  };
  hipError_t e = hipErrorInvalidValue;
  if (p.waves == 0) {
    const int32_t grid = padded_grid(io);
    const DenseRowsSrc<32> src = fill(DenseRowsSrc<32>{});
    if (p.sets == 0 && a.d == 128) hipLaunchKernelGGL((attn_q4_few_kernel<128>), dim3(grid), dim3(kRowWaves * 64), 0, stream, io, src);
    else if (p.sets == 0) hipLaunchKernelGGL((attn_q4_few_kernel<64>), dim3(grid), dim3(kRowWaves * 64), 0, stream, io, src);
    else if (a.d == 128) hipLaunchKernelGGL((attn_q4_rows_kernel<128>), dim3(grid), dim3(kRowWaves * 64), 0, stream, io, src);
    else hipLaunchKernelGGL((attn_q4_rows_kernel<64>), dim3(grid), dim3(kRowWaves * 64), 0, stream, io, src);
    e = hipGetLastError();
  } else {
    const DenseRowsSrc<64> src = fill(DenseRowsSrc<64>{});
#define SV_DENSE(DD, NN, KK) \
  if (a.d == DD && p.waves == NN && p.sets == KK) e = launch_one<DD, NN, KK>(io, src, stream);
    SV_DENSE(64, 2, 4) SV_DENSE(64, 4, 1) SV_DENSE(64, 4, 2) SV_DENSE(64, 8, 1)
    SV_DENSE(128, 2, 4) SV_DENSE(128, 4, 1) SV_DENSE(128, 4, 2) SV_DENSE(128, 8, 1)
#undef SV_DENSE
  }
  if (e != hipSuccess || p.parts == 1) return e;
  return launch_join_parts(io, a.d, p.parts, a.num_cu, stream);
}

CodesForm sparse_q4_form(const GeoTable& G, int32_t k, int32_t BH, int32_t d, int num_cu) {
  const int32_t tile_q = G.eh[k - 1] * G.ew[k - 1];
  const int nw = waves_for(tile_q);
  const int32_t items = BH * tiles_of(G, k) * ((tile_q + nw * kQPerWave - 1) / (nw * kQPerWave));
  // Tiles of 33 to 64 queries (8 x 8): launches of few waves a SIMD walk their rows in two parts, up to
  // one workgroup a CU in four. us in one, two and four, rows of some 1000 tokens: d = 128, 256 workgroups
  // 32.8 / 24.5 / 23.8, 320 41.7 / 31.4 / 41.7, 512 42.4 / 33.1 / 42.5, 640 45.0 / 47.9 / 61.4; d = 64, 256 24.5 /
  // 17.9 / 17.2, 768 33.2 / 29.3 / 44.0, 896 34.6 / 37.5 / 54.8. Rows of 1400: 256 39.1 / 28.6 / 26.6 and
  // 29.2 / 20.6 / 19.1; of some 300: 25.6 / 20.6 / 20.9 and 19.8 / 15.6 / 15.3.
  int32_t sets = 1;
  if (nw == 2 && items <= (d == 64 ? 3 : 2) * num_cu) sets = items <= num_cu && G.C[k] >= 640 ? 4 : 2;
  return CodesForm{nw, sets, 1};
}

hipError_t launch_sparse_attn_q4(const SparseQ4Args& a, hipStream_t stream) {
  const GeoTable& G = *a.G;
  const int32_t tile_q = G.eh[a.k - 1] * G.ew[a.k - 1], G_k = tiles_of(G, a.k);
  const CodesForm form = sparse_q4_form(G, a.k, a.BH, a.d, a.num_cu);
  const int nw = form.waves;
  const int32_t qpw = nw * kQPerWave, slabs = (tile_q + qpw - 1) / qpw;
  Q4IO io;
  io.q = static_cast<const bf16_bits*>(a.q);
  io.o = static_cast<bf16_bits*>(a.o);
  io.lse = a.lse;
  io.q_bh_stride = a.q_bh_stride;
  io.c = a.c4;
  io.o_rows = G.h[a.k - 1] * G.w[a.k - 1];
  io.n_items = a.BH * G_k * slabs;
  io.swizzle = a.swizzle;
  io.scale_log2 = a.softmax_scale * kLog2e;
  io.part_o = nullptr;
  io.part_ml = nullptr;
  io.rows = a.BH * io.o_rows;
  SparseRowsSrc src;
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
