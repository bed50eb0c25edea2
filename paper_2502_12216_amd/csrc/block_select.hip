// Blocks of a cache that a token may look at most, by a cheap score.
//
// The score of block j for query head h is the largest product that a key inside the
// block's bounds could have with the query, u_hj = sum_d (q_d >= 0 ? q_d hi_jd : q_d lo_jd).
// A group's score of a block is the best of its heads', each counted from that head's
// best block: max_h (u_hj - max_i u_hi).  The products of two bf16 are exact and their sums
// are in 64 bits: where the terms are less than 2^30 apart exact too, whatever their order.
// The bound that does not count has no part in a sum (with q (hi + lo) / 2 + |q| (hi - lo) / 2
// it swallows the other where they are more than 2^44 apart).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "common.hpp"
#include "kernels.hpp"
#include "quant.hpp"

namespace tactic {

// Sums over the 16 lanes of a DPP row of two values per lane, in every lane the total of value
// sl / 8: the first step pairs lanes over the upper lane bit, the lower lane of a pair keeps the first
// value and takes its partner's copy.  (Both partners add the same two numbers, so lanes that end
// on the same value hold the same bits.)
__device__ __forceinline__ double reduce2(const double (&v)[2], int sl) {
  const bool up8 = sl & 8;
  double x = (up8 ? v[1] : v[0]) + dpp<0x140>(up8 ? v[0] : v[1]);
  x += dpp<0x141>(x);
  x += dpp<0x4E>(x);
  return x + dpp<0xB1>(x);
}

// What both forms of the scores have: a.per blocks of one KV head, 16 at a time, the next 16 on their
// way (two to four times as many: 0 to 16% slower for 4 x 2048 blocks of four heads).
struct ScoreRange {
  int64_t j0, j1;           // its blocks
  const uint16_t* bounds;   // of the head's first block
  bool none;
};
__device__ __forceinline__ ScoreRange score_range(const SelectArgs& a) {
  const int g = blockIdx.y, b = blockIdx.z, lb = __builtin_ctz(a.block);
  const int64_t kvb = a.kv_indptr[b], n = seq_tokens(a.kv_indptr, a.seq_len, b);
  const int64_t nb = min((n + a.block - 1) >> lb, a.max_blocks), j0 = (int64_t)blockIdx.x * a.per;
  return {j0, min(nb, j0 + a.per), a.bounds + ((int64_t)g * ((a.total >> lb) + a.B) + first_block(kvb, lb, b)) * (2 * kHeadDim),
          j0 >= nb || nb <= a.budget};  // (all of them are chosen)
}
__device__ __forceinline__ double wide(const uint4& w, int e) {  // the bf16 e of eight (a constant after unrolling)
  const uint32_t u = e < 2 ? w.x : e < 4 ? w.y : e < 6 ? w.z : w.w;
  return (double)(e & 1 ? bf16hi(u) : bf16lo(u));
}

// 8 dimensions of a query head in 64 bits, and ones where they are negative
__device__ __forceinline__ void signed_query(const uint16_t* p, double (&q)[8], uint32_t (&neg)[4]) {
  const uint4 w = *reinterpret_cast<const uint4*>(p);
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int e = 0; e < 8; ++e) q[e] = wide(w, e);
#pragma unroll
  for (int i = 0; i < 4; ++i) neg[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(i16x2, u[i]) >> 15);
}
// A lane's part of u_hj from its 8 dimensions of the block's bounds
__device__ __forceinline__ double score_of_lane(const double (&q)[8], const uint32_t (&neg)[4], const uint4& lo, const uint4& hi) {
  auto pick = [](uint32_t m, uint32_t x, uint32_t y) { return (x & m) | (y & ~m); };
  const uint4 w = make_uint4(pick(neg[0], lo.x, hi.x), pick(neg[1], lo.y, hi.y), pick(neg[2], lo.z, hi.z), pick(neg[3], lo.w, hi.w));
  double u = 0.0;
#pragma unroll
  for (int e = 0; e < 8; ++e) u = fma(q[e], wide(w, e), u);
  return u;
}

// One or two query heads, on the vector unit: 16 lanes have a block, 8 dimensions each, and take of
// every two dimensions what the query's signs say before they make 64 bits of it.  A block is 512
// bytes and 128 G conversions and fused operations.  65536 blocks of one head 7.7 us (4.4 TB/s and the
// start), of two 8.4; by the matrix unit, as below, 9.5 both.
template <int G>
__global__ __launch_bounds__(256) void block_score_kernel(SelectArgs a) {
  static_assert(G == 1 || G == 2, "four and eight heads: block_score_matrix_kernel");
  constexpr int kSpan = 16 / G;  // a head's score ends in kSpan lanes
  __shared__ double s_top[16][G];
  const int tid = threadIdx.x, sl = tid & 15, sub = tid >> 4;
  const ScoreRange r = score_range(a);
  if (r.none) return;
  const int64_t head = (int64_t)blockIdx.z * a.Hq + blockIdx.y * G;
  auto load = [&](int64_t j, uint4& lo, uint4& hi) __attribute__((always_inline)) {
    const uint16_t* p = r.bounds + min(j + sub, r.j1 - 1) * (2 * kHeadDim) + sl * 8;
    lo = *reinterpret_cast<const uint4*>(p);
    hi = *reinterpret_cast<const uint4*>(p + kHeadDim);
  };
  uint4 lo, hi, lo2, hi2;
  load(r.j0, lo, hi);
  double q[G][8], best = -INFINITY;
  uint32_t neg[G][4];
#pragma unroll
  for (int h = 0; h < G; ++h) signed_query(a.q + (head + h) * kHeadDim + sl * 8, q[h], neg[h]);
  double* scores = a.scores + (head + sl / kSpan) * a.max_blocks;
#pragma unroll 1
  for (int64_t j = r.j0; j < r.j1; j += 16) {
    load(min(j + 16, r.j1 - 1), lo2, hi2);
    double u[G];
#pragma unroll
    for (int h = 0; h < G; ++h) u[h] = score_of_lane(q[h], neg[h], lo, hi);
    double v;
    if constexpr (G == 2) v = reduce2(u, sl);
    else v = sum16d(u[0]);
    if (j + sub < r.j1) {
      best = fmax(best, v);  // (NaN is passed over, and stored as what it counts as)
      if (sl % kSpan == 0) scores[j + sub] = v != v ? INFINITY : v;
    }
    lo = lo2;
    hi = hi2;
  }
  if (sl % kSpan == 0) s_top[sub][sl / kSpan] = best;
  __syncthreads();
  if (tid < G) {
    double v = s_top[0][tid];
#pragma unroll
    for (int i = 1; i < 16; ++i) v = fmax(v, s_top[i][tid]);
    a.top[(head + tid) * a.tops + blockIdx.x] = v;
  }
}

// 8 dimensions of a query head in 64 bits, its positive and its negative values apart
__device__ __forceinline__ void parts_of_query(const uint16_t* p, double (&above)[8], double (&below)[8]) {
  const uint4 w = *reinterpret_cast<const uint4*>(p);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const double x = wide(w, e);
    above[e] = x < 0 ? 0.0 : x;
    below[e] = x < 0 ? x : 0.0;
  }
}

// Four or eight query heads, on the matrix unit: v_mfma_f64_4x4x4_4b_f64 for four heads and four blocks at
// a time.  Lane l has block l % 4 and the dimensions 8 (l / 4) .. + 7 of its bounds, one to an
// instruction, and the same dimensions of head l % 4's query, its positive and its negative values
// apart; it receives the sums of head l / 16 and block l % 4 over a quarter of the dimensions (l / 4 % 4).
// 16 instructions of 16 cycles for each four heads.  65536 blocks of four heads 9.3 us (on the vector unit
// 10.2), of eight 11.2 (15.4).
template <int G>
__global__ __launch_bounds__(256) void block_score_matrix_kernel(SelectArgs a) {
  static_assert(G == 4 || G == 8, "sets of four heads");
  constexpr int S = G / 4;
  __shared__ double s_top[4][G];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 3, row = lane >> 4;
  const ScoreRange r = score_range(a);
  if (r.none) return;
  const int64_t head = (int64_t)blockIdx.z * a.Hq + blockIdx.y * G;
  auto load = [&](int64_t j, uint4& lo, uint4& hi) __attribute__((always_inline)) {
    const uint16_t* p = r.bounds + min(j + wave * 4 + col, r.j1 - 1) * (2 * kHeadDim) + (lane >> 2) * 8;
    lo = *reinterpret_cast<const uint4*>(p);
    hi = *reinterpret_cast<const uint4*>(p + kHeadDim);
  };
  uint4 lo, hi, lo2, hi2;
  load(r.j0, lo, hi);
  double above[S][8], below[S][8], best[S];  // q where it is positive, and where negative
#pragma unroll
  for (int s = 0; s < S; ++s) {
    parts_of_query(a.q + (head + 4 * s + col) * kHeadDim + (lane >> 2) * 8, above[s], below[s]);
    best[s] = -INFINITY;
  }
  double* scores = a.scores + (head + row) * a.max_blocks;
#pragma unroll 1
  for (int64_t j = r.j0; j < r.j1; j += 16) {
    load(min(j + 16, r.j1 - 1), lo2, hi2);
    double high[S] = {}, low[S] = {};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const double x = wide(lo, e), y = wide(hi, e);
#pragma unroll
      for (int s = 0; s < S; ++s) {
        high[s] = __builtin_amdgcn_mfma_f64_4x4x4f64(above[s][e], y, high[s], 0, 0, 0);
        low[s] = __builtin_amdgcn_mfma_f64_4x4x4f64(below[s][e], x, low[s], 0, 0, 0);
      }
    }
    const int64_t at = j + wave * 4 + col;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      double v = high[s] + low[s];
      v += dpp<0x128>(v);  // row_ror:8 and :4, the quarters of the dimensions
      v += dpp<0x124>(v);
      if (at < r.j1) {
        best[s] = fmax(best[s], v);
        if ((lane & 12) == 0) scores[4 * s * a.max_blocks + at] = v != v ? INFINITY : v;
      }
    }
    lo = lo2;
    hi = hi2;
  }
#pragma unroll
  for (int s = 0; s < S; ++s) {
    best[s] = fmax(best[s], dpp<0x4E>(best[s]));  // over the quad's four blocks
    best[s] = fmax(best[s], dpp<0xB1>(best[s]));
    if ((lane & 15) == 0) s_top[wave][4 * s + row] = best[s];
  }
  __syncthreads();
  if (tid < G) a.top[(head + tid) * a.tops + blockIdx.x] = fmax(fmax(s_top[0][tid], s_top[1][tid]), fmax(s_top[2][tid], s_top[3][tid]));
}

// Scores (none NaN) as integers that order as they do
__device__ __forceinline__ uint64_t order_key(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  return u >> 63 ? ~u : u | 0x8000000000000000ull;
}

// Largest and smallest of a 32-bit word over the wave, in its last lane, by DPP
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
  auto step = [](uint32_t x, uint32_t y) { return max(x, y); };
  v = step(v, (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x111, 0xF, 0xF, false));
  v = step(v, (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x112, 0xF, 0xF, false));
  v = step(v, (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x114, 0xF, 0xF, false));
  v = step(v, (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x118, 0xF, 0xF, false));
  v = step(v, (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x142, 0xA, 0xF, false));
  return step(v, (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x143, 0xC, 0xF, false));
}

// Where a score lies in the range of the free blocks' scores [-width, 0], as a number that rises with it:
// equal ones are told apart by their keys.  (per_width need not be exact, only the same for all.)
__device__ __forceinline__ uint32_t place_in_range(double score, double per_width) {
  return (uint32_t)fmin(fmax(fma(score, per_width, 4294966784.0), 0.0), 4294967295.0);
}

constexpr int kFusedBlocks = 1024;  // of a workgroup that scores its blocks itself, at most

// The scores of the nb blocks of one KV head into LDS by a workgroup of 1024 threads, 64 blocks side by side, as the
// two kernels above; top: the best of every 16 lanes or of every wave.
template <int H>
__device__ __forceinline__ void score_blocks(const SelectArgs& a, int g, int b, int nb, double (*scores)[kFusedBlocks], double (*top)[8]) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lb = __builtin_ctz(a.block);
  const uint16_t* bounds = a.bounds + ((int64_t)g * ((a.total >> lb) + a.B) + first_block(a.kv_indptr[b], lb, b)) * (2 * kHeadDim);
  const uint16_t* query = a.q + ((int64_t)b * a.Hq + g * H) * kHeadDim;
  auto load = [&](int j, int d, uint4& lo, uint4& hi) __attribute__((always_inline)) {
    const uint16_t* p = bounds + (int64_t)min(j, nb - 1) * (2 * kHeadDim) + d;
    lo = *reinterpret_cast<const uint4*>(p);
    hi = *reinterpret_cast<const uint4*>(p + kHeadDim);
  };
  uint4 lo, hi, lo2, hi2;
  if constexpr (H <= 2) {
    constexpr int kSpan = 16 / H;
    const int sl = tid & 15, sub = tid >> 4;
    load(sub, sl * 8, lo, hi);
    double q[H][8], best = -INFINITY;
    uint32_t neg[H][4];
#pragma unroll
    for (int h = 0; h < H; ++h) signed_query(query + h * kHeadDim + sl * 8, q[h], neg[h]);
#pragma unroll 1
    for (int j = sub; j < nb; j += 64) {
      load(j + 64, sl * 8, lo2, hi2);
      double u[H], v;
#pragma unroll
      for (int h = 0; h < H; ++h) u[h] = score_of_lane(q[h], neg[h], lo, hi);
      if constexpr (H == 2) v = reduce2(u, sl);
      else v = sum16d(u[0]);
      best = fmax(best, v);
      if (sl % kSpan == 0) scores[sl / kSpan][j] = v != v ? INFINITY : v;
      lo = lo2;
      hi = hi2;
    }
    if (sl % kSpan == 0) top[sub][sl / kSpan] = best;
  } else {
    const int col = lane & 3, row = lane >> 4, d = (lane >> 2) * 8;
#pragma unroll 1
    for (int h0 = 0; h0 < H; h0 += 4) {
      load(wave * 4 + col, d, lo, hi);
      double above[8], below[8], best = -INFINITY;
      parts_of_query(query + (h0 + col) * kHeadDim + d, above, below);
#pragma unroll 1
      for (int j = wave * 4; j < nb; j += 64) {
        load(j + 64 + col, d, lo2, hi2);
        double high = 0.0, low = 0.0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          high = __builtin_amdgcn_mfma_f64_4x4x4f64(above[e], wide(hi, e), high, 0, 0, 0);
          low = __builtin_amdgcn_mfma_f64_4x4x4f64(below[e], wide(lo, e), low, 0, 0, 0);
        }
        double v = high + low;
        v += dpp<0x128>(v);
        v += dpp<0x124>(v);
        if (j + col < nb) {
          best = fmax(best, v);
          if ((lane & 12) == 0) scores[h0 + row][j + col] = v != v ? INFINITY : v;
        }
        lo = lo2;
        hi = hi2;
      }
      best = fmax(best, dpp<0x4E>(best));
      best = fmax(best, dpp<0xB1>(best));
      if ((lane & 15) == 0) top[wave][h0 + row] = best;
    }
  }
}

// The `budget` blocks of the largest scores of one KV head, ascending.  A radix selection
// in digits of 11 bits, each with a histogram in LDS of the keys still level, that ends as
// soon as all of the digit that holds the last one are wanted: first over a score's place
// in the range of scores, 32 bits linear (the bits of the scores themselves fill few bins, whose
// counts wait for one another: the first digit of 8192 blocks took 8 us), then, where that
// does not tell, over the scores' bits from the first in which they differ.  Block j is thread
// j mod 1024's; chosen ones find their places by a scan of every wave over the ballots of 64 blocks.
// kPer = 0: the scores lie in the workspace and are gone through 16384 at a time.  kFused: they are made here.
// Bound by its chain of loads, scans and barriers: 188 blocks 4.2 us, 2048 (32 groups) 6.8, 8192 (8
// groups) 11.7, 16384 20.5, 40000 64; with integer keys held in place of scores and a block-wide scan
// of the ballots (two barriers more) 5.5, 7.8, 13.7, 22.8, 79.
template <int kPer, bool kFused = false>
__global__ __launch_bounds__(1024) void block_select_kernel(SelectArgs a) {
  static_assert(!kFused || kPer == 1, "scores in LDS");
  constexpr int kBins = 2048, kThreads = 1024, kHeld = kPer ? kPer : 16, kWords = kHeld * 16;
  __shared__ uint32_t s_hist[kBins];
  __shared__ double s_best[8];
  __shared__ double s_scores[kFused ? 8 : 1][kFusedBlocks], s_top[kFused ? 64 : 1][8];
  __shared__ uint32_t s_max[16];
  __shared__ uint64_t s_least[16], s_most[16];
  __shared__ uint32_t s_wave[16];
  __shared__ uint32_t s_digit, s_above, s_in;
  __shared__ __align__(16) uint32_t s_words[kWords];  // chosen and level blocks of each 64
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int g = blockIdx.x, b = blockIdx.y;
  const int lb = __builtin_ctz(a.block), G = a.G;
  const int64_t n = seq_tokens(a.kv_indptr, a.seq_len, b);
  const int nb = (int)min((n + a.block - 1) >> lb, a.max_blocks), want = min(a.budget, nb);
  int32_t* out = a.blocks + ((int64_t)b * a.Hkv + g) * a.budget;
  if (tid == 0) a.counts[(int64_t)b * a.Hkv + g] = want;
  for (int i = want + tid; i < a.budget; i += kThreads) out[i] = -1;
  if (nb <= a.budget) {
    for (int i = tid; i < want; i += kThreads) out[i] = i;
    return;
  }
  const double* scores = a.scores + ((int64_t)b * a.Hq + g * G) * a.max_blocks;
  double* stored = a.keys + ((int64_t)b * a.Hkv + g) * a.max_blocks;
  // the first and the last blocks are chosen whatever their scores: they take no part in the selection
  const int begin = min(a.first, nb), end = max(begin, nb - a.last), forced = nb - (end - begin);
  auto free_block = [&](int j) { return j >= begin && j < end; };
  double held[kHeld];
  uint32_t place[kHeld];
  uint32_t width = 0;  // the least finite score, its size as the bits of a float
  auto all_scores = [&](auto heads) __attribute__((always_inline)) {
    constexpr int H = decltype(heads)::value, K = kHeld < 4 ? kHeld : 4;
    double d[H][K], from[H];
    auto load = [&](int j) __attribute__((always_inline)) {  // K blocks, all loads first
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int i = 0; i < K; ++i) {
          const int at = min(j + i * kThreads, nb - 1);
          if constexpr (kFused) d[h][i] = s_scores[h][at];
          else d[h][i] = scores[(int64_t)h * a.max_blocks + at];
        }
    };
    if constexpr (kFused) {
      score_blocks<H>(a, g, b, nb, s_scores, s_top);
      __syncthreads();
    }
    load(tid);  // (on their way while the best ones are looked up)
    if (wave < H) {  // every head's best score: a wave for each
      double v = -INFINITY;
      if constexpr (kFused) {
        if (lane < (H <= 2 ? 64 : 16)) v = s_top[lane][wave];
      } else {
        const double* top = a.top + ((int64_t)b * a.Hq + g * H + wave) * a.tops;
        for (int i = lane; i < (nb + a.per - 1) / a.per; i += kWave) v = fmax(v, top[i]);
      }
      v = wave_allmax_d(v);
      if (lane == 0) s_best[wave] = v;
    }
    for (int i = tid; i < kBins; i += kThreads) s_hist[i] = 0;
    __syncthreads();
    bool finite = true;  // else a difference may be NaN, which counts as +inf
#pragma unroll
    for (int h = 0; h < H; ++h) {
      from[h] = s_best[h];
      finite &= fabs(from[h]) < INFINITY;
    }
    for (int c = 0; c < nb; c += kHeld * kThreads) {  // (once with kPer)
#pragma unroll
      for (int i = 0; i < kHeld; i += K) {
        if (c + i * kThreads >= nb) break;
        if (c + i > 0) load(c + i * kThreads + tid);
#pragma unroll
        for (int k = 0; k < K; ++k) {
          double best = d[0][k] - from[0];
          if (finite) {
#pragma unroll
            for (int h = 1; h < H; ++h) best = fmax(best, d[h][k] - from[h]);
          } else {
            bool odd = best != best;
#pragma unroll
            for (int h = 1; h < H; ++h) {
              const double y = d[h][k] - from[h];
              odd |= y != y;
              best = fmax(best, y);
            }
            best = odd ? INFINITY : best;
          }
          best += 0.0;  // (-0 as 0)
          held[i + k] = best;
          const int j = c + (i + k) * kThreads + tid;
          const float x = -(float)best;
          if (free_block(j) && x < INFINITY) width = max(width, __float_as_uint(fmaxf(x, 0.f)));
          if constexpr (kPer == 0) {  // (read back by the thread that wrote it)
            if (j < nb) stored[j] = best;
          }
        }
      }
      if constexpr (kPer > 0) break;
    }
  };
  switch (G) {
    case 1: all_scores(std::integral_constant<int, 1>{}); break;
    case 2: all_scores(std::integral_constant<int, 2>{}); break;
    case 4: all_scores(std::integral_constant<int, 4>{}); break;
    default: all_scores(std::integral_constant<int, 8>{}); break;
  }
  width = wave_max_u32(width);
  if (lane == kWave - 1) s_max[wave] = width;
  __syncthreads();
  width = s_max[0];
#pragma unroll
  for (int w = 1; w < 16; ++w) width = max(width, s_max[w]);
  // (neither 0 nor infinite, for a score of +inf to lie above all and one of 0 above the others)
  const float unit = fminf(fmaxf(__builtin_amdgcn_rcpf(__uint_as_float(width)), 0x1p-126f), 0x1p126f);
  const double per_width = 4294966784.0 * (double)unit;
  // f(score, place) of this thread's free blocks
  auto fetch = [&](int c) __attribute__((always_inline)) {
    if constexpr (kPer == 0) {
#pragma unroll
      for (int i = 0; i < kHeld; ++i) held[i] = stored[min(c + i * kThreads + tid, nb - 1 - (nb - 1 - tid) % kThreads)];
#pragma unroll
      for (int i = 0; i < kHeld; ++i) place[i] = place_in_range(held[i], per_width);
    }
  };
  auto each = [&](auto f) __attribute__((always_inline)) {
    for (int c = 0; c < nb; c += kHeld * kThreads) {
      fetch(c);
#pragma unroll
      for (int i = 0; i < kHeld; ++i) {
        if (c + i * kThreads >= nb) break;
        if (free_block(c + i * kThreads + tid)) f(held[i], place[i]);
      }
      if constexpr (kPer > 0) break;
    }
  };
  if constexpr (kPer > 0) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i) place[i] = place_in_range(held[i], per_width);
  }
  uint32_t need = (uint32_t)(want - forced);  // wanted of the free blocks that are level so far
  bool all = need == 0;
  // a digit: counts of the level keys' digits, and the one that holds the last wanted key
  auto digit = [&](auto digit_of) __attribute__((always_inline)) -> uint32_t {
    each([&](double x, uint32_t p) {
      const int d = digit_of(x, p);
      if (d >= 0) atomicAdd(&s_hist[d], 1u);
    });
    __syncthreads();
    // thread t: bins 2 t and 2 t + 1 counted from the top
    const uint32_t c0 = s_hist[kBins - 1 - 2 * tid], c1 = s_hist[kBins - 2 - 2 * tid];
    const uint32_t incl = wave_incl_scan(c0 + c1);
    if (lane == 63) s_wave[wave] = incl;
    s_hist[kBins - 1 - 2 * tid] = 0;  // for the next digit
    s_hist[kBins - 2 - 2 * tid] = 0;
    __syncthreads();
    const uint32_t of_wave = s_wave[lane & 15];  // (a row of 16 lanes scans the waves)
    const uint32_t ahead = (uint32_t)__builtin_amdgcn_readlane((int)(row_incl_scan(of_wave) - of_wave), __builtin_amdgcn_readfirstlane(wave)) + incl - c0 - c1;
    if (ahead < need && ahead + c0 >= need) {
      s_digit = kBins - 1 - 2 * tid;
      s_above = ahead;
      s_in = c0;
    } else if (ahead + c0 < need && ahead + c0 + c1 >= need) {
      s_digit = kBins - 2 - 2 * tid;
      s_above = ahead + c0;
      s_in = c1;
    }
    __syncthreads();
    need -= s_above;
    all = s_in == need;
    return s_digit;
  };
  // places agree above bit `low` with `prefix`
  int low = 32;
  uint32_t prefix = 0;
  while (!all && low > 0) {
    const int bits = min(low, 11), shift = low - bits;
    const uint32_t d = digit([&](double, uint32_t p) {
      return low == 32 || p >> low == prefix ? (int)(p >> shift & ((1u << bits) - 1)) : -1;
    });
    prefix = prefix << bits | d;
    low = shift;
  }
  auto level = [&](uint32_t p) { return low == 32 || p >> low == prefix; };
  // the level keys agree above bit `key_low` with `key_prefix` (64: nothing said of them)
  int key_low = 64;
  uint64_t key_prefix = 0;
  if (!all) {
    uint64_t least = ~0ull, most = 0;
    each([&](double x, uint32_t p) {
      if (level(p)) {
        least = min(least, order_key(x));
        most = max(most, order_key(x));
      }
    });
    for (int d = 32; d >= 1; d /= 2) {
      least = min(least, (uint64_t)__shfl_xor((unsigned long long)least, d, 64));
      most = max(most, (uint64_t)__shfl_xor((unsigned long long)most, d, 64));
    }
    if (lane == 0) {
      s_least[wave] = least;
      s_most[wave] = most;
    }
    __syncthreads();
    for (int w = 0; w < 16; ++w) {
      least = min(least, s_least[w]);
      most = max(most, s_most[w]);
    }
    key_low = least == most ? 0 : 64 - __clzll((long long)(least ^ most));
    key_prefix = key_low >= 64 ? 0 : most >> key_low;
    while (!all && key_low > 0) {
      const int bits = min(key_low, 11), shift = key_low - bits;
      const uint32_t d = digit([&](double x, uint32_t p) {
        const uint64_t k = order_key(x);
        return level(p) && (key_low >= 64 || k >> key_low == key_prefix) ? (int)(k >> shift & ((1u << bits) - 1)) : -1;
      });
      key_prefix = key_low >= 64 ? (uint64_t)d : key_prefix << bits | d;
      key_low = shift;
    }
  }
  // chosen: the blocks that always are, those above the prefixes, and of those level with them the first `need`
  uint32_t done_above = 0, done_same = 0;
  for (int c = 0; c < nb; c += kHeld * kThreads) {
    fetch(c);
    uint64_t above[kHeld], same[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      above[i] = same[i] = 0;
      if (c + i * kThreads < nb) {
        const int j = c + i * kThreads + tid;
        const bool is_free = free_block(j), on = level(place[i]);
        const uint64_t k = key_low >= 64 ? 0 : order_key(held[i]) >> key_low;
        const bool over = (low < 32 && place[i] >> low > prefix) || (on && k > key_prefix);
        above[i] = __ballot(j < nb && (!is_free || (over && want > forced)));
        same[i] = __ballot(is_free && on && k == key_prefix);
      }
      if (lane == 0) s_words[i * 16 + wave] = __popcll(above[i]) | __popcll(same[i]) << 16;
    }
    __syncthreads();
    // counts before each 64 blocks, by every wave for itself: lane l has words W l .. W l + W - 1
    constexpr int W = kWords > 64 ? kWords / 64 : 1;
    uint32_t before_mine = 0, sum = 0;  // (before the word of this wave among a lane's)
    if (W * lane < kWords) {
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const uint32_t c = s_words[W * lane + i];
        before_mine += i < wave % W ? c : 0;
        sum += c;
      }
    }
    const uint32_t incl = wave_incl_scan(sum);
    const int total = __builtin_amdgcn_readlane((int)incl, 63), word = __builtin_amdgcn_readfirstlane(wave / W);
    before_mine += incl - sum;
    const uint64_t before = (1ull << lane) - 1;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      if ((above[i] | same[i]) == 0) continue;  // (the wave has none)
      const uint32_t ahead = (uint32_t)__builtin_amdgcn_readlane((int)before_mine, i * (16 / W) + word);
      const uint32_t at = done_above + (ahead & 0xffff) + __popcll(above[i] & before);
      const uint32_t level_at = done_same + (ahead >> 16) + __popcll(same[i] & before);
      if ((above[i] >> lane & 1) || ((same[i] >> lane & 1) && level_at < need)) out[at + min(level_at, need)] = c + i * kThreads + tid;
    }
    done_above += total & 0xffff;
    done_same += (uint32_t)total >> 16;
    if constexpr (kPer > 0) break;
    __syncthreads();
  }
}

hipError_t launch_block_scores(const SelectArgs& a, hipStream_t st) {
  const dim3 grid((uint32_t)a.tops, a.Hkv, a.B);
  switch (a.G) {
    case 1: hipLaunchKernelGGL((block_score_kernel<1>), grid, dim3(256), 0, st, a); break;
    case 2: hipLaunchKernelGGL((block_score_kernel<2>), grid, dim3(256), 0, st, a); break;
    case 4: hipLaunchKernelGGL((block_score_matrix_kernel<4>), grid, dim3(256), 0, st, a); break;
    case 8: hipLaunchKernelGGL((block_score_matrix_kernel<8>), grid, dim3(256), 0, st, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

// Whether the workgroup that selects scores its blocks itself.  A rule for eager calls, where a second launch takes 2
// us more of the host; replayed from a graph the two meet at fewer blocks.  us a call in one launch and in two, eager |
// replayed: 4 groups of one head 256 blocks 6.5, 8.7 | 6.2, 6.1; 512 8.0, 8.6 | 7.7, 6.3; of two heads 192 7.3, 8.5 | 7.0, 6.6;
// 256 8.0, 8.6 | 7.7, 6.6; 320 8.5, 8.7 | 8.1, 6.6; of four 128 6.9, 8.7 | 6.6, 6.6; 160 7.8, 8.6 | 7.5, 6.6; 192 8.0, 9.4 | 7.6, 7.1;
// of eight 48 7.3, 9.6 | 6.9, 7.6; 64 8.1, 9.5 | 7.8, 7.6; 128 10.1, 9.6 | 9.7, 7.9; 32 groups of four 160 7.9, 8.5 | 7.6, 7.6; 192
// 8.6, 8.4 | 8.2, 7.5; 224 9.0, 8.3 | 8.7, 7.4; of eight 64 8.3, 8.6 | 8.0, 7.8; 80 9.1, 8.7 | 8.8, 8.1.  256 groups, a compute unit
// each, where the GPU's time counts in both: of one head 1024 blocks 22.6, 26.5; of four 23.9, 29.2; of eight 512 23.9,
// 25.2; 768 32.9, 32.5.
bool blocks_scored_by_select(const SelectArgs& a) {
  if ((int64_t)a.B * a.Hkv >= 256) return a.max_blocks <= (a.G == 8 ? 512 : kFusedBlocks);
  return a.max_blocks <= (a.G == 8 ? 64 : a.G == 4 ? 192 : 256);
}

hipError_t launch_block_select(const SelectArgs& a, hipStream_t st) {
  const dim3 grid(a.Hkv, a.B), threads(1024);
  if (blocks_scored_by_select(a)) hipLaunchKernelGGL((block_select_kernel<1, true>), grid, threads, 0, st, a);
  else if (a.max_blocks <= 1024) hipLaunchKernelGGL((block_select_kernel<1>), grid, threads, 0, st, a);
  else if (a.max_blocks <= 2048) hipLaunchKernelGGL((block_select_kernel<2>), grid, threads, 0, st, a);
  else if (a.max_blocks <= 4096) hipLaunchKernelGGL((block_select_kernel<4>), grid, threads, 0, st, a);
  else if (a.max_blocks <= 8192) hipLaunchKernelGGL((block_select_kernel<8>), grid, threads, 0, st, a);
  else if (a.max_blocks <= kSelectHeld) hipLaunchKernelGGL((block_select_kernel<16>), grid, threads, 0, st, a);
  else hipLaunchKernelGGL((block_select_kernel<0>), grid, threads, 0, st, a);
  return hipGetLastError();
}

}  // namespace tactic
