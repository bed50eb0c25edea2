// Attention of many query rows over one key sequence on the matrix unit: the
// prompt form (the rows are the G heads of consecutive tokens) and the shared
// prefix of a decode batch (the rows are the G heads of the sequences that
// share it).
//
// A work item is a row tile (32 rows for each of RW waves) of one KV head and a
// range of its keys, in tiles of TK.  A wave computes S^T = K Q^T with
// v_mfma_f32_32x32x16_bf16, so that a lane's accumulators belong to one query
// row (column lane % 32) and the running maximum and sum of the softmax need one
// exchange, with lane ^ 32.  The weights of 16 keys in a lane are then the B
// operand of O^T += V^T P^T as they stand: the matrix unit sums over keys, so
// their order is free as long as V^T has the same, and the transposing LDS read
// (ds_read_b64_tr_b16) gives four consecutive keys of one dimension, which is the
// order the accumulators of S^T have.  KW groups of waves take every KW-th tile
// and are merged at the end; where there are few items their keys are split and
// joined by rows_combine_kernel (the shared prefix by combine_kernel), in a fixed order.
//
// Weights go to the matrix unit as bf16 where the output is bf16 (half a step of
// each, 2^-8, as the output's own rounding; sums in 32 bits), in three parts that hold
// all 24 bits where it is fp32.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "common.hpp"
#include "kernels.hpp"
#include "scores.hpp"

namespace tactic {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// LDS rows are 16 chunks of 16 bytes; logical chunk c of row r is stored at chunk
// c ^ row_swizzle(r): 16 consecutive rows at one chunk (the K operand) and 4 rows
// of 4 chunks (the transposing V read) both fall in distinct banks.
__device__ __forceinline__ int row_swizzle(int r) { return 4 * (r & 3) + ((r >> 2) & 3); }

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const f32x2 x = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}

// Eight weights as the bf16 operands of PARTS products.  1: rounded to nearest
// (outputs in bf16: off by at most 2^-8 of a weight, as the output's own
// rounding).  3: an exact split of the fp32 weight for outputs in fp32; the lower
// parts of a weight that is not zero are at least 2^-126, so that its product with
// an infinite value stays that infinity.
template <int PARTS>
__device__ __forceinline__ void weight_operands(const float (&p)[8], u32x4 (&out)[PARTS]) {
  if constexpr (PARTS == 1) {
#pragma unroll
    for (int i = 0; i < 4; ++i) out[0][i] = pack_bf16(p[2 * i], p[2 * i + 1]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t h[2], m[2], l[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float x = p[2 * i + j], least = fminf(x, 0x1p-126f);
        h[j] = __float_as_uint(x);
        const float r = x - __uint_as_float(h[j] & 0xffff0000u);
        m[j] = __float_as_uint(fmaxf(r, least));
        l[j] = __float_as_uint(fmaxf(r - __uint_as_float(__float_as_uint(r) & 0xffff0000u), least));
      }
      out[0][i] = __builtin_amdgcn_perm(h[1], h[0], 0x07060302u);
      out[1][i] = __builtin_amdgcn_perm(m[1], m[0], 0x07060302u);
      out[2][i] = __builtin_amdgcn_perm(l[1], l[0], 0x07060302u);
    }
  }
}

// Which halves of a word, under `mask`, lie in [lo, lo + span]: 0x3f80 (1.0) there, 0 elsewhere.
__device__ __forceinline__ uint32_t halves_in(uint32_t w, uint32_t mask, uint32_t lo, uint32_t span) {
  const uint32_t a = ((w & mask) - lo) <= span ? 0x3f80u : 0u, b = (((w >> 16) & mask) - lo) <= span ? 0x3f800000u : 0u;
  return a | b;
}
__device__ __forceinline__ uint32_t finite_halves(uint32_t w) {
  const uint32_t lo = (w & 0x7f80u) == 0x7f80u ? 0u : 0xffffu, hi = (w & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u;
  return w & (lo | hi);
}

// Maximum and sum of the values of lanes l and l ^ 32, the same in both.
__device__ __forceinline__ float halves_max(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);  // the lower half's value, the upper's
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float halves_sum(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Row in the pages of token `tok` of sequence b (in bounds whatever the table holds;
// the host has checked that the pages hold fewer than 2^31 rows).  `shift`: log2 of the
// page size, or negative.
__device__ __forceinline__ int page_row(const PagedKV& pk, int shift, int Hkv, int b, int kvh, int tok) {
  const uint32_t pg = shift >= 0 ? (uint32_t)tok >> shift : (uint32_t)tok / (uint32_t)pk.page_size;
  const int page = min(max(pk.page_table[(int64_t)b * pk.max_pages + pg], 0), (int)pk.num_pages - 1);
  return (page * Hkv + kvh) * pk.page_size + (tok - (int)(pg * (uint32_t)pk.page_size));
}

constexpr float kMaxFinite = 3.402823466e38f;  // a score of +inf: the sum becomes inf (its logarithm too), the output NaN
constexpr float kRescaleSlack = 8.f;  // base-2: a weight may exceed 1 by 2^8 before the sums are rescaled

// Source of row tile `rest`: the tiles of source b start at floor(rows before it / rows)
// + b at the latest.  A lane per candidate, 64 at a time: one load where there are few.
__device__ __forceinline__ int source_of(const RowsArgs& a, int rows, int rest, int lane) {
  int src = 0;
  for (int count = a.n_src; count > 1;) {
    const int step = (count + 63) / 64, mid = src + lane * step;
    bool ok = lane * step < count;
    if (ok) {
      const int64_t before = a.mode == 0 ? a.q_indptr[mid] : (int64_t)a.member_indptr[mid];
      ok = before * a.G / rows + mid <= rest;
    }
    const int at = ((int)__popcll(__ballot(ok)) - 1) * step;  // (candidate 0 always is)
    src += at;
    count = min(step, count - at);
  }
  return src;
}
// Range of the documents of tokens [p0, p1] of a sequence, from those of its 64-token
// tiles (at most 5 of them), the same in all lanes.  Empty where p1 < 0.
__device__ __forceinline__ int2 docs_of(const int2* dr, int p0, int p1, int lane) {
  int lo = INT32_MAX, hi = INT32_MIN;
  if (p1 >= 0 && p0 / 64 + lane <= p1 / 64) {
    const int2 r = dr[p0 / 64 + lane];
    lo = r.x;
    hi = r.y;
  }
#pragma unroll
  for (int s = 1; s < 8; s <<= 1) {
    lo = min(lo, __shfl_xor(lo, s, 64));
    hi = max(hi, __shfl_xor(hi, s, 64));
  }
  return make_int2(__builtin_amdgcn_readfirstlane(lo), __builtin_amdgcn_readfirstlane(hi));
}

// RW waves hold 32 rows each and share a tile of keys, KW such groups take turns at the
// tiles.  The host takes 32, 64, 128 or 256 rows to an item by an estimate of the time
// (plan_rows, with the measurements).  Bound by the matrix unit where a prompt is long:
// 16384 tokens, 32 heads on 8, take 2060 to 2140 us (1.03 to 1.07 PFLOP/s; a library
// product of 8192^3 reaches 1.11), 2250 to 2320 with slopes, 2480 to 2540 with a cap, whose polynomial
// competes with the exponential for the vector unit.  512 tokens on 65536 in pages, with
// slopes: 609 us, 0.90 PFLOP/s.  Packed documents (29193 tokens, 1100 on average, cap):
// 800 us, 0.60: the tiles hold 1.09 of the pairs that count, the cap takes a sixth, each item's
// start and end 12 of its 84 us (the chain from the item's record to the first keys, the waves'
// last turn), the kernels ahead 14, the tiles masked in part (16%) and uneven ends the rest.  A prefix of 32768 tokens and 32
// sequences: 47 us, by the matrix unit (the weights' three parts make the products twice as
// many) and HBM (2.9 TB/s) together.
template <int RW, int KW, int TK, int PARTS, bool kPaged, bool kDocs>
__global__ __launch_bounds__(RW * KW * 64) __attribute__((amdgpu_waves_per_eu(2)))
void rows_attn_kernel(RowsArgs a) {
  constexpr int ROWS = RW * 32, NW = RW * KW, NB = TK / 32;
  constexpr int kBufs = RW > 1 ? 2 : 1;                  // one wave alone reads and writes its tile in turn
  constexpr int kTileBytes = TK * 256 * 2;               // K rows, then V rows
  constexpr int kLoads = TK * 16 / (RW * 64);            // 16-byte chunks of K (and of V) per thread and tile
  constexpr int kStage = KW * kBufs * kTileBytes, kMerge = KW > 1 ? NW * 16384 : 0;
  __shared__ __align__(1024) unsigned char smem[kStage > kMerge ? kStage : kMerge];
  __shared__ float s_ml[2][NW][32];
  __shared__ __align__(16) int s_doc[kDocs ? KW * kBufs * TK : 4];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave % RW, kg = wave / RW, half = lane >> 5, col = lane & 31;

  // ---- the work item: KV head (fastest, so that a head's items share an XCD's L2
  // where 8 divides the heads), split, row tile of a source
  const int g = blockIdx.x % a.Hkv;
  int rest = blockIdx.x / a.Hkv;
  const int split = rest % a.splits;
  rest /= a.splits;
  int src, i_lo = INT32_MAX, i_hi = INT32_MIN;  // and the documents of the item's queries
  const bool ordered = kDocs && RW == 8 && a.order;  // (only the form of 256 rows is started in order)
  if (ordered) {
    const int4 item = a.order[rest];
    rest = item.x;
    src = item.y;
    i_lo = item.z;
    i_hi = item.w;
  } else {
    src = source_of(a, ROWS, rest, lane);
  }
  const int64_t q0 = a.mode == 0 ? a.q_indptr[src] : (int64_t)a.member_indptr[src];
  const int64_t q1 = a.mode == 0 ? a.q_indptr[src + 1] : (int64_t)a.member_indptr[src + 1];
  const int nrows = (int)((q1 - q0) * a.G);
  const int ntile = (nrows + ROWS - 1) / ROWS;
  int tile = rest - (int)(q0 * a.G / ROWS) - src;
  if (tile < 0 || tile >= ntile) return;
  tile = ntile - 1 - tile;  // the last rows of a prompt see the most keys: first
  const int row0 = tile * ROWS;
  const int64_t kvb = a.kv_indptr[src];
  const int n = (int)seq_tokens(a.kv_indptr, a.seq_len, src);

  // ---- this lane's row (rows past the end repeat the last one and are not stored)
  const int row = min(row0 + wr * 32 + col, nrows - 1);
  const bool own_row = row0 + wr * 32 + col < nrows;
  const int h = row % a.G;
  int64_t qrow;         // row of q, out and lse: query * Hq + head
  int qpos, klim = n;   // keys [0, klim) are seen
  int qdoc = 0;
  if (a.mode == 0) {
    const int i = row / a.G;
    const int64_t m = q1 - q0;
    qrow = (q0 + i) * a.Hq + g * a.G + h;
    qpos = (int)(n - m + i);
    const int pre = a.prefix_len ? a.prefix_len[src] : 0;
    klim = min(max(max(qpos + 1, pre), 0), n);
    if (kDocs) qdoc = qpos >= 0 ? a.documents[kvb + qpos] : 0;
    if (qpos < 0) klim = 0;  // more queries than tokens: those ahead of the first see nothing
  } else {
    const int b = a.members[q0 + row / a.G];
    qrow = (int64_t)b * a.Hq + g * a.G + h;
    qpos = n + (int)seq_tokens(a.own_indptr, a.own_len, b) - 1;
  }
  // the item's keys: those that its last row sees (prompt rows see ever more)
  int kend = n, kall = n;  // and those that its first row sees
  if (a.mode == 0) {
    const int last = min(row0 + ROWS, nrows) - 1;
    const int lp = (int)(n - (q1 - q0) + last / a.G);
    const int pre = a.prefix_len ? a.prefix_len[src] : 0;
    kend = lp < 0 ? 0 : min(max(lp + 1, pre), n);
    const int fp = (int)(n - (q1 - q0) + row0 / a.G);
    kall = fp < 0 ? 0 : min(max(fp + 1, pre), n);
  }
  const int ktiles = (kend + TK - 1) / TK;
  const int t_lo = (int)((int64_t)ktiles * split / a.splits), t_hi = (int)((int64_t)ktiles * (split + 1) / a.splits);

  // the fewest keys that one of the wave's rows sees (rows ascend)
  const int w_lo = __builtin_amdgcn_readlane(klim, 0);

  // Scores without a cap stay a factor `scale` below their base-2 value until the
  // exponential, which takes it along with the maximum in one multiply-add.
  const bool capped = a.cap > 0.f, biased = a.slopes != nullptr;
  const float scale = capped ? 1.f : kInvSqrtDim * kLog2e;
  const float slope = biased ? a.slopes[g * a.G + h] * kLog2e / scale : 0.f;
  const float to_cap = capped ? kInvSqrtDim / a.cap : 0.f, cap2 = a.cap * kLog2e;

  bf16x8 qf[8];
  auto load_q = [&]() __attribute__((always_inline)) {
    const uint16_t* qp = a.q + qrow * kHeadDim + 8 * half;
#pragma unroll
    for (int s = 0; s < 8; ++s) qf[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(qp + 16 * s));
  };
  load_q();

  // Documents: ranges of each 64-key tile (from doc_range_kernel).  i_lo, i_hi: of the
  // tiles that the item's queries lie in; a tile outside is left out by the forms of 32
  // and 256 rows, and masked by the others, whose groups of waves go by fixed rounds (8192
  // tokens, 8 heads on 2, documents of 300: 237 us, 178 without documents).  Ranges are read
  // 64 tiles at a time, into masks of the tiles that may hold a seen key, of those whose
  // keys all are of the wave's one document, and of those where that holds for the item.
  const int2* dr = kDocs ? a.doc_range + (int64_t)src * a.range_stride : nullptr;
  int win = INT32_MIN;
  uint64_t w_some = 0, w_same = 0, w_sure = 0;
  const int d_one = __builtin_amdgcn_readfirstlane(qdoc);
  const bool one_doc = __all(qdoc == d_one);
  if (kDocs && !ordered) {
    const int64_t m = q1 - q0;
    const int2 r = docs_of(dr, max((int)(n - m + row0 / a.G), 0), (int)(n - m + (min(row0 + ROWS, nrows) - 1) / a.G), lane);
    i_lo = r.x;
    i_hi = r.y;
  }
  auto look = [&](int t) __attribute__((always_inline)) {
    if (t >= win && t < win + 64) return;
    win = t;
    int2 r = make_int2(INT32_MAX, INT32_MIN);
    if (t + lane < t_hi) r = dr[(t + lane) * TK / 64];
    w_some = __ballot(r.x <= i_hi && r.y >= i_lo);
    w_same = __ballot(one_doc && r.x == r.y && r.x == d_one);
    w_sure = __ballot(i_lo == i_hi && r.x == r.y && r.x == i_lo);
  };
  // first tile from t on, in steps of KW, that may hold a seen key (t_hi or more: none)
  constexpr uint64_t kEvery = KW == 1 ? ~0ull : (KW == 2 ? 0x5555555555555555ull : 0x1111111111111111ull);
  auto next_tile = [&](int t) __attribute__((always_inline)) -> int {
    if constexpr (!kDocs) return t;
    while (t < t_hi) {
      look(t);
      const uint64_t any = (w_some >> (t - win)) & kEvery;
      if (any) return t + __ffsll((unsigned long long)any) - 1;
      t += (win + 64 - t + KW - 1) / KW * KW;
    }
    return t;
  };
  // whether all of the wave's rows see all of the tile (kFull), and all of the item's (kSure)
  constexpr int kFull = 1, kSure = 2;
  auto sees_all = [&](int t) __attribute__((always_inline)) -> int {
    int all = (t * TK + TK <= w_lo ? kFull : 0) | (t * TK + TK <= kall ? kSure : 0);
    if constexpr (kDocs) {
      if (t < t_hi) {
        look(t);
        all &= (int)(w_same >> (t - win) & 1) | (int)(w_sure >> (t - win) & 1) << 1;
      }
    }
    return all;
  };

  const uint16_t* Kb = a.K + (kPaged ? 0 : ((int64_t)g * a.total + kvb) * kHeadDim);
  const uint16_t* Vb = a.V + (kPaged ? 0 : ((int64_t)g * a.total + kvb) * kHeadDim);
  u32x4 kreg[kLoads], vreg[kLoads];
  int doc_r = 0;
  // chunk i of this thread: stored chunk (wr * kLoads + i) * 64 + lane of the group's tile
  const int doc_wave = RW == 8 ? 4 : 0;
  const int f_row = wr * kLoads * 4 + (lane >> 4), f_swz = row_swizzle(f_row), f_col = lane & 15;
  // element offset of chunk i of tile t: in token order a constant beside the tile's
  // own (a scalar), in pages by the table
  auto rows_of = [&](int t, int (&at)[kLoads]) __attribute__((always_inline)) {
    const int most = n - 1 - t * TK;  // rows past the end repeat the last
#pragma unroll
    for (int i = 0; i < kLoads; ++i) at[i] = (t + 1) * TK <= n ? f_row + 4 * i : min(f_row + 4 * i, most);
  };
  // rows of the pages (paged only)
  const int page_shift = kPaged && (a.pk.page_size & (a.pk.page_size - 1)) == 0 ? 31 - __clz(a.pk.page_size) : -1;
  auto page_rows_of = [&](int t, int (&row)[kLoads]) __attribute__((always_inline)) {
    int at[kLoads];
    rows_of(t, at);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) row[i] = page_row(a.pk, page_shift, a.Hkv, src, g, t * TK + at[i]);
  };
  auto load_paged = [&](const uint16_t* base, const int (&row)[kLoads], u32x4 (&reg)[kLoads]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      reg[i] = *reinterpret_cast<const u32x4*>(base + (int64_t)row[i] * kHeadDim + ((f_col ^ f_swz ^ (i & 3)) * 8));
  };
  auto load = [&](const uint16_t* base, int t, u32x4 (&reg)[kLoads]) __attribute__((always_inline)) {
    int at[kLoads];
    if constexpr (kPaged) {
      page_rows_of(t, at);
      load_paged(base, at, reg);
    } else {
      rows_of(t, at);
      const unsigned char* tile_base = reinterpret_cast<const unsigned char*>(base + (int64_t)t * (TK * kHeadDim));
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        reg[i] = *reinterpret_cast<const u32x4*>(tile_base + (uint32_t)(at[i] * 256 + ((f_col ^ f_swz ^ (i & 3)) * 16)));
    }
  };
  auto fetch_doc = [&](int t) __attribute__((always_inline)) {
    if constexpr (kDocs) {
      if (wr == doc_wave && lane < TK) doc_r = a.documents[kvb + min(t * TK + lane, n - 1)];
    }
  };
  auto fetch_k = [&](int t) __attribute__((always_inline)) {
    load(Kb, t, kreg);
    fetch_doc(t);
  };
  auto fetch_v = [&](int t) __attribute__((always_inline)) { load(Vb, t, vreg); };
  auto place = [&](int buf) __attribute__((always_inline)) {
    return smem + (kg * kBufs + buf) * kTileBytes + (wr * kLoads * 64 + lane) * 16;
  };
  auto store_k = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) *reinterpret_cast<u32x4*>(place(buf) + i * 1024) = kreg[i];
    if constexpr (kDocs) {
      if (wr == doc_wave && lane < TK) s_doc[(kg * kBufs + buf) * TK + lane] = doc_r;
    }
  };
  auto store_v = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) *reinterpret_cast<u32x4*>(place(buf) + i * 1024 + TK * 256) = vreg[i];
  };
  auto fetch = [&](int t) __attribute__((always_inline)) {
    if constexpr (kPaged) {
      int row[kLoads];
      page_rows_of(t, row);
      load_paged(Kb, row, kreg);
      load_paged(Vb, row, vreg);
      fetch_doc(t);
    } else {
      fetch_k(t);
      fetch_v(t);
    }
  };
  auto store = [&](int buf) __attribute__((always_inline)) {
    store_k(buf);
    store_v(buf);
    if constexpr (RW == 1) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // one wave writes and reads the tile
  };

  float m_run = -INFINITY, l4[4] = {0.f, 0.f, 0.f, 0.f};
  f32x16 o[4];
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.f;

  // LDS offsets of the operands.  K: row col (+ 32 kb), chunk 2 st + half.  V: two
  // transposing reads of 4 keys per operand of 16 keys and 32 dimensions; lane l of a
  // group of 16 gives the address of row l / 4, 8-byte piece l % 4.  The constant parts
  // of a chunk enter the swizzled place by exclusive or.
  const uint32_t k_off = col * 256 + ((half ^ row_swizzle(col)) * 16);
  const int v_row = 4 * half + ((lane & 15) >> 2);
  const uint32_t v_off = v_row * 256 + (((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ row_swizzle(v_row)) * 16) + (lane & 1) * 8;
  typedef __attribute__((address_space(3))) unsigned char* lds_ptr;
  typedef __attribute__((address_space(3))) s16x4* lds4_ptr;

  auto tile_lds = [&](int buf) __attribute__((always_inline)) { return (lds_ptr)(smem + (kg * kBufs + buf) * kTileBytes); };

  f32x16 s[NB];           // scores of the tile, then dead
  u32x4 pf[TK / 16][PARTS];  // its weights
  // Operands are read a step ahead of their products and no further (sched_barrier):
  // left to itself the compiler reads the whole tile ahead and spills the rows in flight.
  // `beside(step)` is work to place between the products of every second step.
  auto qk = [&](int buf, auto beside) __attribute__((always_inline)) {
    const lds_ptr kt = tile_lds(buf);
    uint32_t off = k_off;
    asm volatile("" : "+v"(off));  // (its eight places are made here, not kept in registers over the loop)
    typedef __attribute__((address_space(3))) u32x4* lds16_ptr;
    u32x4 kf[2][NB];
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) {
      kf[0][kb] = *(lds16_ptr)(kt + kb * 8192 + off);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
    }
#pragma unroll
    for (int st = 0; st < 8; ++st) {
      if (st < 7) {
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) kf[(st + 1) & 1][kb] = *(lds16_ptr)(kt + kb * 8192 + (off ^ ((st + 1) * 32)));
      }
#pragma unroll
      for (int kb = 0; kb < NB; ++kb)
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[st & 1][kb]), qf[st], s[kb], 0, 0, 0);
      if (st & 1) {
        beside(st / 2);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  auto nothing = [](int) __attribute__((always_inline)) {};

  // scores to weights; accumulator r of block kb is key k0 + 32 kb + 8 (r / 4) + 4 half + r % 4
  auto soft = [&](int t, int buf, bool masked, bool dead) __attribute__((always_inline)) {
    const int k0 = t * TK;
    if (capped) {
      float big = 0.f;
#pragma unroll
      for (int kb = 0; kb < NB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) big = fmaxf(big, fabsf(s[kb][r]));
      // (NaN counts as inside: the polynomials keep it)
      if (PARTS == 1 && !__any(big > a.poly.near)) {
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            s[kb][r] = cap_near(s[kb][r], a.poly);
            if (r % 8 == 7) __builtin_amdgcn_sched_barrier(0);
          }
      } else if (!__any(big > a.poly.far)) {
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            s[kb][r] = cap_far(s[kb][r], a.poly);
            if (r % 8 == 7) __builtin_amdgcn_sched_barrier(0);
          }
      } else {
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            s[kb][r] = cap2 * tanh_any(s[kb][r] * to_cap);
            if (r % 2) __builtin_amdgcn_sched_barrier(0);  // (two at a time: few registers are left here)
          }
      }
    }
    if (biased) {
      const float dist = (float)(qpos - k0 - 4 * half);
#pragma unroll
      for (int kb = 0; kb < NB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          s[kb][r] = fmaf(-slope, fabsf(dist - (float)(kb * 32 + 8 * (r / 4) + r % 4)), s[kb][r]);
    }
    if (masked) {
      const int lim = dead ? 0 : klim - k0 - 4 * half;  // (dead: nothing of the tile counts)
#pragma unroll
      for (int kb = 0; kb < NB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (kb * 32 + 8 * (r / 4) + r % 4 >= lim) s[kb][r] = -INFINITY;
      if constexpr (kDocs) {
        const int* dk = s_doc + (kg * kBufs + buf) * TK + 4 * half;
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; r += 4) {
            const int4 d = *reinterpret_cast<const int4*>(dk + kb * 32 + 2 * r);
            s[kb][r] = d.x != qdoc ? -INFINITY : s[kb][r];
            s[kb][r + 1] = d.y != qdoc ? -INFINITY : s[kb][r + 1];
            s[kb][r + 2] = d.z != qdoc ? -INFINITY : s[kb][r + 2];
            s[kb][r + 3] = d.w != qdoc ? -INFINITY : s[kb][r + 3];
          }
      }
    }
    float m4[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) m4[j] = s[0][j];
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
      for (int r = kb == 0 ? 4 : 0; r < 16; ++r) m4[r & 3] = fmaxf(m4[r & 3], s[kb][r]);
    float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
    mx = halves_max(mx) * scale;
    // the sums keep an old maximum as their reference while no weight exceeds 2^8
    if (__any(mx > m_run + kRescaleSlack)) {
      const float mn = fminf(fmaxf(mx, m_run), kMaxFinite);
      const float c = mn > m_run ? fast_exp2(m_run - mn) : 1.f;
      m_run = mn;
#pragma unroll
      for (int j = 0; j < 4; ++j) l4[j] *= c;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= c;
    }
    const float ref = m_run == -INFINITY ? 0.f : m_run;
#pragma unroll
    for (int c = 0; c < TK / 16; ++c) {
      float p[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        p[j] = fast_exp2(fmaf(s[c / 2][8 * (c % 2) + j], scale, -ref));
        l4[j & 3] += p[j];
      }
      weight_operands<PARTS>(p, pf[c]);
    }
#pragma unroll
    for (int c = 0; c < TK / 16; ++c)
#pragma unroll
      for (int k = 0; k < PARTS; ++k) asm volatile("" : "+v"(pf[c][k]));  // (made here, before the barrier, not at their use)
#pragma unroll
    for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(l4[j]));
  };

  auto v_operand = [&](lds_ptr vt, uint32_t off, int c, int d) __attribute__((always_inline)) -> u32x4 {
    const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4_ptr)(vt + c * 4096 + (off ^ (d * 64)))));
    const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4_ptr)(vt + c * 4096 + 2048 + (off ^ (d * 64 + 32)))));
    return u32x4{x.x, x.y, y.x, y.y};
  };
  auto pv = [&](int buf) __attribute__((always_inline)) {
    const lds_ptr vt = tile_lds(buf) + TK * 256;
    uint32_t off = v_off;
    asm volatile("" : "+v"(off));
    u32x4 vf[2][4];
#pragma unroll
    for (int d = 0; d < 4; ++d) vf[0][d] = v_operand(vt, off, 0, d);
#pragma unroll
    for (int c = 0; c < TK / 16; ++c) {
      if (c + 1 < TK / 16) {
#pragma unroll
        for (int d = 0; d < 4; ++d) vf[(c + 1) & 1][d] = v_operand(vt, off, c + 1, d);
      }
#pragma unroll
      for (int k = PARTS - 1; k >= 0; --k)
#pragma unroll
        for (int d = 0; d < 4; ++d)
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[c & 1][d]), __builtin_bit_cast(bf16x8, pf[c][k]), o[d], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // A masked key's weight is 0, but 0 times its value is NaN where that is not
  // finite.  So the values of tiles with something masked are looked over, a part by
  // each wave of the tile, and where one is found the item is computed again by a loop
  // that goes by kinds of values.
  auto any_odd = [&](int buf) __attribute__((always_inline)) -> bool {
    constexpr int kPart = TK * 16 / 64 / RW;
    const lds_ptr vt = tile_lds(buf) + TK * 256 + wr * kPart * 1024;
    uint32_t bad = 0;
#pragma unroll
    for (int i = 0; i < kPart; ++i) {
      const u32x4 w = *(__attribute__((address_space(3))) u32x4*)(vt + (i * 64 + lane) * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) bad |= w[j] ^ finite_halves(w[j]);
    }
    return __any(bad != 0);
  };
  auto pv_odd = [&](int t, int buf) __attribute__((always_inline)) {
    const lds_ptr vt = tile_lds(buf) + TK * 256;
    // which keys the row sees, by the masks: a weight may be 0 without one (bit r + 16 kb as
    // in soft; by arithmetic and four at a time, since the masks of comparisons and more
    // registers here are spilled by the loops above: 128 rows with documents in pages, 3001
    // tokens, 32 heads on 8, 218 us that way, 196 now, 193 where a weight of 0 counted as masked)
    static_assert(NB <= 2, "a bit per key");
    const int lim = klim - t * TK - 4 * half;
    uint32_t seen = 0;
#pragma unroll 1
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll 1
      for (int r = 0; r < 16; r += 4) {
        uint32_t in = (1u << min(max(lim - kb * 32 - 2 * r, 0), 4)) - 1u;
        if constexpr (kDocs) {
          const int4 d = *reinterpret_cast<const int4*>(s_doc + (kg * kBufs + buf) * TK + 4 * half + kb * 32 + 2 * r);
          const uint32_t other = min((uint32_t)(d.x ^ qdoc), 1u) | min((uint32_t)(d.y ^ qdoc), 1u) << 1 |
                                 min((uint32_t)(d.z ^ qdoc), 1u) << 2 | min((uint32_t)(d.w ^ qdoc), 1u) << 3;
          in &= ~other;
        }
        seen |= in << (kb * 16 + r);
      }
    // finite values as in pv; then, for each kind of value that is not finite, whether a
    // seen key has it in this dimension: an infinity (1, 2) with a weight, NaN (3), an
    // infinity without a weight, which gives NaN as 0 times it does in pv (4)
#pragma unroll
    for (int c = 0; c < TK / 16; ++c)
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        u32x4 w = v_operand(vt, v_off, c, d);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = finite_halves(w[j]);
#pragma unroll
        for (int k = PARTS - 1; k >= 0; --k)
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, pf[c][k]), o[d], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);  // one operand at a time: few registers are left here
      }
#pragma unroll 1
    for (int kind = 1; kind < 5; ++kind) {
      const float val = kind == 1 ? INFINITY : (kind == 2 ? -INFINITY : NAN);
      const uint32_t mask = kind >= 3 ? 0x7fffu : 0xffffu, lo = kind == 2 ? 0xff80u : (kind == 3 ? 0x7f81u : 0x7f80u),
                     span = kind == 3 ? 0x7eu : 0u;
      const uint32_t by_weight = kind < 3 ? ~0u : 0u, no_weight = kind == 4 ? ~0u : 0u;
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        f32x16 hit;
#pragma unroll
        for (int r = 0; r < 16; ++r) hit[r] = 0.f;
#pragma unroll
        for (int c = 0; c < TK / 16; ++c) {
          u32x4 w = v_operand(vt, v_off, c, d), one;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            w[j] = halves_in(w[j], mask, lo, span);
            const uint32_t weight = ((pf[c][0][j] & 0xffffu) ? 0x3f80u : 0u) | ((pf[c][0][j] & 0xffff0000u) ? 0x3f800000u : 0u);
            const uint32_t bits = seen >> (8 * c + 2 * j), sees = (bits & 1u) * 0x3f80u | (bits >> 1 & 1u) * 0x3f800000u;
            one[j] = (weight & by_weight) | (sees & ~by_weight & ~(weight & no_weight));
          }
          hit = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, one), hit, 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] += hit[r] != 0.f ? val : 0.f;
      }
    }
  };
  bool odd = false;

  // ---- the keys
  if constexpr (RW * KW == 8) {
    // Eight waves, two per SIMD, take turns: while waves 0 to 3 do the products of a
    // tile (P V of the one before, then K Q), waves 4 to 7 turn scores into weights,
    // and the other way round, a barrier between.  In phase 2 i waves 0 to 3 contract
    // their tile i, in phase 2 i + 1 the others do.  Each brings its part of K of tile
    // i + 1 and V of tile i to LDS there, between the products (a block of its own took
    // 470 of a phase's 2200 cycles): into the buffers of
    // tiles i - 1 and i - 2, whose last reads are in phase 2 i - 1, for first reads in
    // phase 2 i + 2.  (Documents are read with the weights, in phases 2 i + 1 and
    // 2 i + 2: where all waves share the tiles a late wave brings them.)  KW = 1: all
    // waves go by one list of tiles.  Else group kg takes tile first + kg of each round
    // of KW, and one past the end is the last one again, masked as a whole.
    constexpr bool kOne = KW == 1;
    auto round = [&](int t) __attribute__((always_inline)) { return kOne ? next_tile(t) : t; };
    auto of = [&](int t) __attribute__((always_inline)) { return kOne ? t : min(t + kg, t_hi - 1); };
    int t = round(t_lo);
    if (t < t_hi) {
      const bool late = wave >= 4;
      // tiles of this round and the next ones, and whether no row masks any of them
      // (past the end of the list: dead, and masked as a whole)
      auto whole = [&](int t) __attribute__((always_inline)) -> int { return t + kg < t_hi ? sees_all(of(t)) : 0; };
      int full0 = whole(t);
      int t1 = round(t + KW);
      int full1 = whole(t1);
      fetch_k(of(t));
      store_k(0);
      fetch_v(of(t));
      // pages: the rows of a tile are looked up a round before its keys are fetched, and
      // serve its values a round later (rows1: of t1, rows2: of the tile after)
      int rows1[kLoads], rows2[kLoads], t2 = t1;
      if (t1 < t_hi) t2 = round(t1 + KW);
      int full2 = whole(t2);
      if constexpr (kPaged) {
        page_rows_of(of(min(t1, t_hi - 1)), rows1);
        load_paged(Kb, rows1, kreg);
        fetch_doc(of(min(t1, t_hi - 1)));
        page_rows_of(of(min(t2, t_hi - 1)), rows2);
      } else {
        fetch_k(of(min(t1, t_hi - 1)));
      }
      __syncthreads();
      if (late) __syncthreads();
      int i = 0;
      bool look_over;
      for (;;) {
        int t3 = t2;
        if (t2 < t_hi) t3 = round(t2 + KW);
        const int full3 = whole(t3);
        // (past the end the last tile is brought again, which nobody reads)
        const int tv = of(min(t1, t_hi - 1)), tk = of(min(t2, t_hi - 1)), tr = of(min(t3, t_hi - 1));
        qk(i & 1, [&](int step) __attribute__((always_inline)) {
          if (step == 0) store_v(i & 1);
          if (step == 1) store_k((i + 1) & 1);
          if constexpr (kPaged) {
            if (step == 2) load_paged(Vb, rows1, vreg);
            if (step == 3) {
              load_paged(Kb, rows2, kreg);
              fetch_doc(tk);
#pragma unroll
              for (int j = 0; j < kLoads; ++j) rows1[j] = rows2[j];
              page_rows_of(tr, rows2);
            }
          } else {
            if (step == 2) fetch_v(tv);
            if (step == 3) fetch_k(tk);
          }
        });
        __syncthreads();
        const bool dead = !kOne && t + kg >= t_hi;
        look_over = !(full0 & kSure);
        soft(of(t), i & 1, !(full0 & kFull), dead);
        t = t1;
        t1 = t2;
        t2 = t3;
        full0 = full1;
        full1 = full2;
        full2 = full3;
        if (!(late && t >= t_hi)) __syncthreads();  // (the late waves have made one more)
        if (look_over) odd |= any_odd(i & 1);
        if (t >= t_hi) break;
        pv(i & 1);
        ++i;
      }
      pv(i & 1);
    }
  } else {
    // each wave by itself: the next tile's rows are in flight while this one is contracted
    static_assert(RW == 1, "waves that share a tile take turns");
    int t = next_tile(t_lo + kg);
    if (t < t_hi) {
      fetch(t);
      store(0);
    }
    while (t < t_hi) {
      const int tn = next_tile(t + KW);
      if (tn < t_hi) fetch(tn);
      const bool masked = !(sees_all(t) & kFull);
      qk(0, nothing);
      soft(t, 0, masked, false);
      if (masked) odd |= any_odd(0);
      pv(0);
      if (tn < t_hi) store(0);
      t = tn;
    }
  }
  if (__syncthreads_or(odd)) {  // rare: the whole item again, one tile at a time
    m_run = -INFINITY;
#pragma unroll
    for (int j = 0; j < 4; ++j) l4[j] = 0.f;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
    load_q();
#pragma unroll 1
    for (int t0 = t_lo; t0 < t_hi; t0 += KW) {
      const int t = t0 + kg;
      if (t < t_hi) {
        fetch(t);
        store(0);
      }
      __syncthreads();
      if (t < t_hi) {
        qk(0, nothing);
        soft(t, 0, !(sees_all(t) & kFull), false);
        pv_odd(t, 0);
      }
      __syncthreads();
    }
  }

  // ---- the sums of both halves, then of the KW groups
  float l_run = halves_sum((l4[0] + l4[1]) + (l4[2] + l4[3]));
  // (a maximum passes NaN over: where no other score was there the sum says that some was)
  if (m_run == -INFINITY && l_run != l_run) m_run = 0.f;
  int d_from = 0, d_to = 4;
  if constexpr (KW > 1) {
    __syncthreads();  // the tiles are dead: their storage takes the groups' sums
    if (half == 0) {
      s_ml[0][wave][col] = m_run;
      s_ml[1][wave][col] = l_run;
    }
    __syncthreads();
    float mm = -INFINITY, ll = 0.f;
#pragma unroll
    for (int j = 0; j < KW; ++j) mm = fmaxf(mm, s_ml[0][j * RW + wr][col]);
#pragma unroll
    for (int j = 0; j < KW; ++j) {
      const float mj = s_ml[0][j * RW + wr][col];
      if (mj != -INFINITY) ll = fmaf(s_ml[1][j * RW + wr][col], fast_exp2(mj - mm), ll);
    }
    const float c = m_run == -INFINITY ? 0.f : fast_exp2(m_run - mm);
    float* red = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) red[(wave * 64 + d * 16 + r) * 64 + lane] = m_run == -INFINITY ? 0.f : o[d][r] * c;
    __syncthreads();
    m_run = mm;
    l_run = ll;
    d_from = kg * (4 / KW);
    d_to = d_from + 4 / KW;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      if (d < d_from || d >= d_to) continue;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float x = 0.f;
#pragma unroll
        for (int j = 0; j < KW; ++j) x += red[((j * RW + wr) * 64 + d * 16 + r) * 64 + lane];
        o[d][r] = x;
      }
    }
  }
  if (!own_row) return;
  if (a.direct) {
    const float inv = l_run != 0.f ? 1.f / l_run : 0.f;  // (NaN stays NaN)
    uint16_t* op = a.out + qrow * kHeadDim + 4 * half;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      if (d < d_from || d >= d_to) continue;
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        u32x2 w = {pack_bf16(o[d][r] * inv, o[d][r + 1] * inv), pack_bf16(o[d][r + 2] * inv, o[d][r + 3] * inv)};
        *reinterpret_cast<u32x2*>(op + d * 32 + 2 * r) = w;
      }
    }
    if (a.lse && kg == 0 && half == 0) {
      const int64_t hq = qrow % a.Hq, qi = qrow / a.Hq;
      a.lse[hq * a.n_queries + qi] = m_run == -INFINITY ? -INFINITY : (m_run + __builtin_amdgcn_logf(l_run)) * kLn2;
    }
  } else {
    const int64_t slot = (int64_t)split * a.n_queries * a.Hq + qrow;
    float* op = a.part_o + slot * kHeadDim + 4 * half;
    if (m_run != -INFINITY) {
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        if (d < d_from || d >= d_to) continue;
#pragma unroll
        for (int r = 0; r < 16; r += 4)
          *reinterpret_cast<float4*>(op + d * 32 + 2 * r) = make_float4(o[d][r], o[d][r + 1], o[d][r + 2], o[d][r + 3]);
      }
    }
    if (kg == 0 && half == 0) {
      a.part_ml[2 * slot] = m_run;
      a.part_ml[2 * slot + 1] = l_run;
    }
  }
}

// Range of the documents of every 64-row tile: grid (tiles, sequences), one wave each.
__global__ __launch_bounds__(64) void doc_range_kernel(const int32_t* documents, const int64_t* kv_indptr,
                                                       const int64_t* seq_len, int64_t stride, int2* out) {
  const int b = blockIdx.y, t = blockIdx.x;
  const int n = (int)seq_tokens(kv_indptr, seq_len, b);
  if (t * 64 >= n) return;
  const int32_t d = documents[kv_indptr[b] + min(t * 64 + (int)threadIdx.x, n - 1)];
  int lo = d, hi = d;
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    lo = min(lo, __shfl_xor(lo, s, 64));
    hi = max(hi, __shfl_xor(hi, s, 64));
  }
  if (threadIdx.x == 0) out[b * stride + t] = make_int2(lo, hi);
}

// Key tiles (of 64) that each row tile's queries may see: what its documents leave of
// them.  A wave per row tile.
__global__ __launch_bounds__(256) void doc_items_kernel(RowsArgs a, int tiles, int4* items, int32_t* counts) {
  constexpr int rows = 256;  // of an item
  const int lane = threadIdx.x & 63, rest = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (rest >= tiles) return;
  const int src = source_of(a, rows, rest, lane);
  const int64_t q0 = a.q_indptr[src], m = a.q_indptr[src + 1] - q0;
  const int nrows = (int)(m * a.G), ntile = (nrows + rows - 1) / rows;
  const int tile = ntile - 1 - (rest - (int)(q0 * a.G / rows) - src);  // (as in rows_attn_kernel)
  int count = 0;
  int2 own = make_int2(INT32_MAX, INT32_MIN);
  if (tile >= 0 && tile < ntile) {
    const int n = (int)seq_tokens(a.kv_indptr, a.seq_len, src);
    const int2* dr = a.doc_range + (int64_t)src * a.range_stride;
    const int p0 = max((int)(n - m + tile * rows / a.G), 0), p1 = (int)(n - m + (min(tile * rows + rows, nrows) - 1) / a.G);
    own = docs_of(dr, p0, p1, lane);
    const int kend = p1 < 0 ? 0 : min(max(p1 + 1, a.prefix_len ? a.prefix_len[src] : 0), n), kt = (kend + 63) / 64;
    for (int t = lane; t < kt; t += 64) {
      const int2 r = dr[t];
      count += r.x <= own.y && r.y >= own.x;
    }
  }
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) count += __shfl_xor(count, s, 64);
  if (lane == 0) {
    items[rest] = make_int4(rest, src, own.x, own.y);
    counts[rest] = count;
  }
}
// The row tiles by falling count, in 32 steps of the largest, in their own order within
// a step: long ones started last would end after all others (documents of 100 to 8000
// tokens: the last fifth of the time had idle units), and neighbours share their keys in
// L2.  One workgroup, a wave for two steps, the counts in LDS (460 row tiles: 9 us,
// bound by its chain; doc_items_kernel 5).
__global__ __launch_bounds__(1024) void item_order_kernel(const int4* items, const int32_t* counts, int tiles, int4* order) {
  constexpr int kHeld = 8192;  // counts of the first tiles, read again by every wave
  __shared__ int s_most[16], s_count[32], s_held[kHeld];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int most = 1;
  for (int t = threadIdx.x; t < tiles; t += 1024) {
    const int c = counts[t];
    if (t < kHeld) s_held[t] = c;
    most = max(most, c);
  }
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) most = max(most, __shfl_xor(most, s, 64));
  if (lane == 0) s_most[wave] = most;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 16; ++w) most = max(most, s_most[w]);
  const float inv = 1.f / (float)most;
  auto step_of = [&](int t) __attribute__((always_inline)) -> int {  // 0: the longest; -1: none
    return t < tiles ? 31 - (int)((float)(t < kHeld ? s_held[t] : counts[t]) * 31.f * inv) : -1;
  };
  int n0 = 0, n1 = 0;
  for (int t = 0; t < tiles; t += 64) {
    const int s = step_of(t + lane);
    n0 += __popcll(__ballot(s == 2 * wave));
    n1 += __popcll(__ballot(s == 2 * wave + 1));
  }
  if (lane == 0) {
    s_count[2 * wave] = n0;
    s_count[2 * wave + 1] = n1;
  }
  __syncthreads();
  int at0 = 0;
  for (int s = 0; s < 2 * wave; ++s) at0 += s_count[s];
  int at1 = at0 + n0;
  for (int t = 0; t < tiles; t += 64) {
    const int s = step_of(t + lane);
    const uint64_t in0 = __ballot(s == 2 * wave), in1 = __ballot(s == 2 * wave + 1), before = (1ull << lane) - 1;
    if (s == 2 * wave) order[at0 + __popcll(in0 & before)] = items[t + lane];
    if (s == 2 * wave + 1) order[at1 + __popcll(in1 & before)] = items[t + lane];
    at0 += __popcll(in0);
    at1 += __popcll(in1);
  }
}

// Joins the splits of a row: out = sum_s O_s 2^(m_s - M) / sum_s l_s 2^(m_s - M).  One
// wave per row: lane s has split s's maximum and sum, so that M and the sum of the
// weights are wave reductions (in one order); then two dimensions per lane, eight
// splits' sums in flight.
__global__ __launch_bounds__(256) void rows_combine_kernel(RowsArgs a) {
  const int64_t rows = a.n_queries * a.Hq;
  const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (r >= rows) return;
  static_assert(kMaxSplits <= kWave, "a lane per split");
  float m = -INFINITY, l = 0.f;
  if (lane < a.splits) {
    const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + 2 * ((int64_t)lane * rows + r));
    m = ml.x;
    l = ml.y;
  }
  const float* po = a.part_o + r * kHeadDim + 2 * lane;
  const float mx = wave_allmax_f(m);
  const float c = m == -INFINITY ? 0.f : fast_exp2(m - mx);  // (a split without keys wrote no sums)
  l = wave_allsum_f(m == -INFINITY ? 0.f : l * c);
  const uint64_t some = __ballot(m != -INFINITY);
  float x = 0.f, y = 0.f;
#pragma unroll 8
  for (int s = 0; s < a.splits; ++s) {
    if (!(some >> s & 1)) continue;
    const float2 v = *reinterpret_cast<const float2*>(po + (int64_t)s * rows * kHeadDim);
    const float w = readlane_f(c, s);
    x = fmaf(v.x, w, x);
    y = fmaf(v.y, w, y);
  }
  const float inv = l != 0.f ? 1.f / l : 0.f;
  *reinterpret_cast<uint32_t*>(a.out + r * kHeadDim + 2 * lane) = pack_bf16(x * inv, y * inv);
  if (a.lse && lane == 0)
    a.lse[(r % a.Hq) * a.n_queries + r / a.Hq] = mx == -INFINITY ? -INFINITY : (mx + __builtin_amdgcn_logf(l)) * kLn2;
}

int rows_per_item(int variant) { return 32 << variant; }

hipError_t launch_doc_range(const int32_t* documents, const int64_t* kv_indptr, const int64_t* seq_len, int batch,
                            int64_t max_tiles, int2* out, hipStream_t st) {
  if (max_tiles == 0) return hipSuccess;
  hipLaunchKernelGGL(doc_range_kernel, dim3((unsigned)max_tiles, batch), dim3(64), 0, st, documents, kv_indptr, seq_len,
                     max_tiles, out);
  return hipGetLastError();
}

hipError_t launch_item_order(const RowsArgs& a, int tiles, int4* items, int32_t* counts, int4* order, hipStream_t st) {
  hipLaunchKernelGGL(doc_items_kernel, dim3((tiles + 3) / 4), dim3(256), 0, st, a, tiles, items, counts);
  hipLaunchKernelGGL(item_order_kernel, dim3(1), dim3(1024), 0, st, items, counts, tiles, order);
  return hipGetLastError();
}

template <int PARTS, bool kPaged, bool kDocs>
static hipError_t launch_rows_t(const RowsArgs& a, int variant, int64_t items, hipStream_t st) {
  const dim3 grid((unsigned)items);
  switch (variant) {
    case 0: hipLaunchKernelGGL((rows_attn_kernel<1, 4, 32, PARTS, kPaged, kDocs>), grid, dim3(256), 0, st, a); break;
    case 1: hipLaunchKernelGGL((rows_attn_kernel<2, 4, 32, PARTS, kPaged, kDocs>), grid, dim3(512), 0, st, a); break;
    case 2: hipLaunchKernelGGL((rows_attn_kernel<4, 2, PARTS == 1 ? 64 : 32, PARTS, kPaged, kDocs>), grid, dim3(512), 0, st, a); break;
    default: hipLaunchKernelGGL((rows_attn_kernel<8, 1, PARTS == 1 ? 64 : 32, PARTS, kPaged, kDocs>), grid, dim3(512), 0, st, a); break;
  }
  return hipGetLastError();
}

hipError_t launch_rows_attn(const RowsArgs& a, int variant, bool exact_weights, int64_t items, hipStream_t st) {
  if (exact_weights) return a.paged ? launch_rows_t<3, true, false>(a, variant, items, st) : launch_rows_t<3, false, false>(a, variant, items, st);
  if (a.documents) return a.paged ? launch_rows_t<1, true, true>(a, variant, items, st) : launch_rows_t<1, false, true>(a, variant, items, st);
  return a.paged ? launch_rows_t<1, true, false>(a, variant, items, st) : launch_rows_t<1, false, false>(a, variant, items, st);
}

hipError_t launch_rows_combine(const RowsArgs& a, hipStream_t st) {
  const int64_t rows = a.n_queries * a.Hq;
  hipLaunchKernelGGL(rows_combine_kernel, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace tactic
