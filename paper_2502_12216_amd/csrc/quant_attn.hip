// One new token per sequence over a quantised cache: all of its rows or those of chosen
// blocks, split over the workgroups and joined by the combine of the dense decode.
//
// A row of K and V is 264 or 136 bytes for 512 G operations: bound by HBM as long as
// codes become products in few instructions.  A wave takes two tiles of 16 rows a step, and
// everything stays in the lanes that loaded it:
//  - Scores: v_mfma_f32_16x16x32_bf16 with the rows of K as the first operand - lane l has
//    row l % 16 and 32 of its dimensions, made bf16 exactly by one conversion for two of
//    them - and four query heads as the columns, repeated four times.  So lane l receives the
//    scores of head l % 4 for the rows 4 (l / 16) .. + 3 of both tiles.
//  - Values: the same instruction with the weights as the first operand: its row l % 16
//    is head l % 4 and the part (l % 16) / 4 of the weight, three bf16 parts whose sum is
//    exact, so that one instruction takes all parts of four heads; its columns are lane l's
//    dimensions 8 (l % 16) .. + 7, one to an instruction, for the same eight rows.
// (The instructions that multiply 8 and 4 bit codes themselves add with fewer bits: 9e-5
// of the absolute sum for a row of 128 codes, where fp32 has 6e-8.)
//
// 4 x 131072 rows, 8 KV heads of 4 query heads: 8 bits 172 us (6.4 TB/s), 4 bits 95 (6.0; 89 of
// them at that rate, the rest the start and the merge; a step of 32 rows is 200 vector and 16 matrix
// instructions, two thirds of the time that its bytes take).  Two waves per SIMD: three spill
// (119 us), one has nothing to run beside its waits (102).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "common.hpp"
#include "kernels.hpp"
#include "plan.hpp"
#include "quant.hpp"
#include "scores.hpp"

namespace tactic {

constexpr float kScaleLog2 = kLog2e * kInvSqrtDim;
// Rows of the least share of a workgroup.  Shares of 128, 192, 256, 384 rows, us a call: 8 bits, 8 KV heads,
// one sequence of 4096 rows 13.2, 11.9, 12.4, 13.9; two of 2300 13.1, 12.0, 12.4, 13.4; 3000 + 2500 with eight
// heads each 15.3, 13.9, 15.9, 17.6; 4 bits, 8192 rows 13.6, 13.3, 12.5, 13.1.
template <int kBits>
constexpr int64_t kQuantShare = kBits == 8 ? 192 : 256;
constexpr int kTableRows = 2048;      // rows looked up at once
// Waves of a workgroup.  Eight: 3 to 11% slower where they split all rows; with a group to itself 5 to 20% slower up to
// 512 rows and 10 to 40% beyond 256 groups, at best 7% faster (128 groups of 2048 rows).
constexpr int kWaves = 4;
constexpr int kStep = 32 * kWaves;    // rows of a step of all of them

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_words __attribute__((aligned(4)));  // (a row's powers begin at any word)

__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// The power of group g of a row from the word of its four bytes: rotated to where a float has
// its exponent, the only part that the conversions read
__device__ __forceinline__ float power_in(uint32_t word, int turn) { return __uint_as_float(__builtin_amdgcn_alignbit(word, word, turn)); }
__device__ __forceinline__ int turn_of(int g) { return 9 + 8 * g; }

template <typename T>
__device__ __forceinline__ T uniform(T x) {
  if constexpr (sizeof(T) == 4) return __builtin_bit_cast(T, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x)));
  else return (T)(((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)((uint64_t)x >> 32)) << 32) | (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
}

// What a workgroup knows of a group: where its sequence's rows begin, the sequence's length, and
// the rows attended: all, or those of its chosen blocks (ascending, so that only the last one
// may be the sequence's last, of fewer rows).
struct Group {
  int64_t kvb;
  int32_t n, rows;
};
__device__ __forceinline__ Group group_of(const QuantAttnArgs& x, int bg) {
  const int b = bg / x.a.NV;
  const int listed = x.blocks ? x.counts[bg] : 0;
  const int64_t kvb = x.a.kv_indptr[b], n = seq_tokens(x.a.kv_indptr, x.a.seq_len, b);
  Group g{kvb, (int32_t)n, (int32_t)n};
  if (x.blocks) {  // (whatever a list holds, the rows are among the sequence's)
    const int lb = __builtin_ctz(x.block);
    const int64_t nb = (n + x.block - 1) >> lb, count = min((int64_t)min(max(listed, 0), x.budget), nb);
    const int64_t last = min(max((int64_t)x.blocks[(int64_t)bg * x.budget + max(count - 1, (int64_t)0)], (int64_t)0), nb - 1);
    g.rows = count == 0 ? 0 : (int32_t)(((count - 1) << lb) + min(n - (last << lb), (int64_t)x.block));
  }
  return g;
}

// kRows: 0 rows lie at their positions; 1 every 16 positions from a multiple of 16 lie together
// (chosen blocks, pages of a multiple of 16 rows); 2 rows lie anywhere
// kDirect: a workgroup for each group, which writes the outputs itself.  (A form of its own: with
// the choice made inside the kernel 5 to 24% slower, and splits with eight heads by up to 14%.)
template <int G, int kBits, int kRows, bool kMod, bool kDirect>
__global__ __launch_bounds__(kWave * kWaves) __attribute__((amdgpu_waves_per_eu(2)))
void quant_attn_kernel(QuantAttnArgs x) {
  constexpr int kPart = G * (kHeadDim + 2);
  constexpr int S = G == 8 ? 2 : 1;           // sets of four heads
  constexpr int RB = kRowBytes<kBits>;
  constexpr int KW = kBits == 8 ? 2 : 1;      // 16-byte words of a lane's dimensions of K
  constexpr int VW = kBits == 8 ? 2 : 1;      // 4-byte words of its 8 values
  constexpr int kThreads = kWave * kWaves;
  const AttnArgs& a = x.a;
  extern __shared__ int64_t s_prefix[];       // [B * NV + 1] units before each group, then [B * NV] the groups
  union Shared {
    struct {
      int tile[kTableRows / 16];              // place of 16 positions (kRows 1)
      int row[kTableRows / 16];               // their rows of the sequence
      __align__(16) int place[kRows == 2 ? kTableRows : 1];
    } t;
    float red[3 * kWaves][G][kHeadDim];       // the merge: three parts of every wave
  };
  __shared__ __align__(16) Shared sh;
  __shared__ float s_ml[kWaves][2][G];
  __shared__ int64_t s_wsum[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int sl = lane & 15, grp = lane >> 4, hd = sl & 3;
  // what a lane takes off its weights: the upper 8 bits from the second part on, the next from the third on
  const uint32_t off1 = sl >= 4 ? 0xffff0000u : 0u, off2 = sl >= 8 ? 0xffff0000u : 0u;
  const int BG = a.B * a.NV;
  // The rows of group bg, [seg_lo, seg_hi): all of them where every group has a workgroup of its
  // own, else this workgroup's share of the units (rows plus the cost of a segment) of all groups,
  // of which segments begin at multiples of 32 rows.
  int bg = blockIdx.x, bg_end = bg + 1;
  int64_t t0 = 0, t1 = INT64_MAX;
  if constexpr (!kDirect) {
    const int per = (BG + kThreads - 1) / kThreads, g0 = min(BG, tid * per), g1 = min(BG, g0 + per);
    auto units = [&](int64_t n) { return n > 0 ? ((n + 31) & ~(int64_t)31) + kSegmentCost : 0; };
    Group* const groups = reinterpret_cast<Group*>(s_prefix + BG + 1);
    int64_t loc = 0;
    for (int g = g0; g < g1; ++g) {
      groups[g] = group_of(x, g);
      loc += units(groups[g].rows);
    }
    const int64_t incl = wave_incl_scan(loc);
    if (lane == kWave - 1) s_wsum[wave] = incl;
    __syncthreads();
    int64_t run = incl - loc;
    for (int w = 0; w < wave; ++w) run += s_wsum[w];
    for (int g = g0; g < g1; ++g) {
      s_prefix[g] = run;
      run += units(groups[g].rows);
    }
    if (tid == kThreads - 1) s_prefix[BG] = run;
    __syncthreads();
    const int64_t total = uniform(s_prefix[BG]);
    // (at least the quotient: its error is far below the least fraction that it can have)
    const int64_t even = (int64_t)((double)total * x.per_grid) + 1;
    const int64_t share = max((even + 31) & ~(int64_t)31, kQuantShare<kBits>);
    if (blockIdx.x == 0) {  // for the combine
      if (tid == 0) a.ameta[0] = share;
      for (int g = tid; g <= BG; g += kThreads) a.ameta[1 + g] = s_prefix[g];
    }
    t0 = (int64_t)blockIdx.x * share;
    t1 = min(total, t0 + share);
    if (t0 >= t1) return;
    // the largest group that starts at or before t0: 64 of them looked at in one step, then those between
    const int stride = (BG + 63) / 64;
    bg = (__popcll(__ballot(lane * stride < BG && s_prefix[min(lane * stride, BG)] <= t0)) - 1) * stride;
    if (stride > 1) bg += __popcll(__ballot(lane < stride && bg + lane < BG && s_prefix[min(bg + lane, BG)] <= t0)) - 1;
    bg = __builtin_amdgcn_readfirstlane(bg);
    bg_end = BG;
  }

  for (; bg < bg_end; ++bg) {
    int64_t seg_lo = 0, seg_hi, kvb;
    int nseq;
    if constexpr (kDirect) {
      const Group g = group_of(x, bg);
      seg_hi = uniform(g.rows);
      kvb = uniform(g.kvb);
      nseq = uniform(g.n);
    } else {
      const int64_t start = uniform(s_prefix[bg]);
      if (start >= t1) break;
      const Group g = reinterpret_cast<const Group*>(s_prefix + BG + 1)[bg];  // (no more loads before the rows')
      seg_lo = max(t0 - start - kSegmentCost, (int64_t)0);
      seg_hi = min((int64_t)uniform(g.rows), t1 - start - kSegmentCost);
      if (seg_lo >= seg_hi) continue;
      kvb = uniform(g.kvb);
      nseq = uniform(g.n);
    }
    const int b = bg / a.NV, kvh = bg % a.NV;

    // the queries, in the dimensions that the lane has of K
    bf16x8 qv[S][4];
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const uint16_t* qp = a.q + ((int64_t)b * a.Hq + kvh * G + (G >= 4 ? 4 * s + hd : hd % G)) * kHeadDim;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        qv[s][j] = *reinterpret_cast<const bf16x8*>(qp + (kBits == 8 ? (j >> 1) * 64 + grp * 16 + (j & 1) * 8 : grp * 32 + j * 8));
    }
    float slope2[S], to_cap = 0.f;
#pragma unroll
    for (int s = 0; s < S; ++s) slope2[s] = 0.f;
    if constexpr (kMod) {
#pragma unroll
      for (int s = 0; s < S; ++s)
        slope2[s] = x.slopes ? x.slopes[kvh * G + (G >= 4 ? 4 * s + hd : hd % G)] * kLog2e : 0.f;
      to_cap = x.cap > 0.f ? kInvSqrtDim / x.cap : 0.f;
    }
    // a head's reference maximum (the same in all lanes of the wave that have the head) and the sum
    // over this lane's rows; sums of values: element i of lane group p is part p of head i
    float m[S], l[S];
    f32x4 acc[S][8];
#pragma unroll
    for (int s = 0; s < S; ++s) {
      m[s] = -3.402823466e38f;
      l[s] = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[s][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int64_t base = x.kv.paged ? 0 : (int64_t)kvh * a.total + kvb;
    const uint8_t* const Kb = x.kv.K + base * RB;
    const uint8_t* const Vb = x.kv.V + base * RB;
    const uint8_t* const Ks = x.kv.K_scale + base * 4;
    const uint8_t* const Vs = x.kv.V_scale + base * 4;
    // the groups of the lane's dimensions
    const int k_turn = kBits == 8 ? turn_of(grp >> 1) : turn_of(grp), k_turn2 = turn_of(2 + (grp >> 1)), v_turn = turn_of(sl >> 2);
    int cnt = 0;
    int64_t p0 = 0;
    struct Tile {
      u32x4 k[2][KW];
      uint32_t v[8][VW];   // rows 4 grp .. + 3 of the first tile, then of the second
      uint32_t ks[2], vs[8];
    };
    auto load_k = [&](Tile& r, int t, const uint8_t* p, const uint8_t* ps) __attribute__((always_inline)) {
#pragma unroll
      for (int w = 0; w < KW; ++w) r.k[t][w] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + 64 * w));
      r.ks[t] = *reinterpret_cast<const uint32_t*>(ps);
    };
    auto load_v = [&](Tile& r, int i, const uint8_t* p) __attribute__((always_inline)) {
      if constexpr (kBits == 8) {
        const u32x2 w = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p));
        r.v[i][0] = w.x;
        r.v[i][1] = w.y;
      } else {
        r.v[i][0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(p));
      }
    };
    // step `step` of this wave: positions kStep step + 32 wave .. + 31 of the sub-range; those
    // past its end read its last row, which the group attends anyway
    auto load_tile = [&](int step) __attribute__((always_inline)) -> Tile {
      Tile r;
      const int at = step * kStep + wave * 32;
      if constexpr (kRows == 2) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int64_t row = sh.t.place[min(at + 16 * t + sl, cnt - 1)];
          load_k(r, t, Kb + row * RB + grp * 16, Ks + row * 4);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int64_t vrow = sh.t.place[min(at + 16 * t + 4 * grp + i, cnt - 1)];
            load_v(r, 4 * t + i, Vb + vrow * RB + sl * (RB / 16));
            r.vs[4 * t + i] = *reinterpret_cast<const uint32_t*>(Vs + vrow * 4);
          }
        }
      } else {
        auto place = [&](int pos) -> int64_t {  // of 16 positions
          if constexpr (kRows == 0) return p0 + pos;
          else return (int64_t)__builtin_amdgcn_readfirstlane(sh.t.tile[pos >> 4]);
        };
        if (at + 32 <= cnt) {
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const int64_t row = place(at + 16 * t);
            load_k(r, t, Kb + row * RB + (uint32_t)(sl * RB + grp * 16), Ks + row * 4 + (uint32_t)(sl * 4));
#pragma unroll
            for (int i = 0; i < 4; ++i) load_v(r, 4 * t + i, Vb + row * RB + (uint32_t)(grp * (4 * RB) + sl * (RB / 16)) + i * RB);
            const u32x4 w = *reinterpret_cast<const u32x4_words*>(Vs + row * 4 + (uint32_t)(grp * 16));
#pragma unroll
            for (int i = 0; i < 4; ++i) r.vs[4 * t + i] = w[i];
          }
        } else {
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const int from = min(at + 16 * t, (cnt - 1) & ~15), most = min(cnt - 1 - from, 15);
            const int64_t row = place(from);
            load_k(r, t, Kb + row * RB + (uint32_t)(min(sl, most) * RB + grp * 16), Ks + row * 4 + (uint32_t)(min(sl, most) * 4));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int in = min(4 * grp + i, most);
              load_v(r, 4 * t + i, Vb + row * RB + (uint32_t)(in * RB + sl * (RB / 16)));
              r.vs[4 * t + i] = *reinterpret_cast<const uint32_t*>(Vs + row * 4 + (uint32_t)(in * 4));
            }
          }
        }
      }
      return r;
    };
    auto consume = [&](const Tile& y, int step) __attribute__((always_inline)) {
      f32x4 d[S][2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const float power = power_in(y.ks[t], k_turn), power2 = power_in(y.ks[t], k_turn2);
#pragma unroll
        for (int s = 0; s < S; ++s) d[s][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          u32x4 w;
          if constexpr (kBits == 8) {
            const uint32_t c0 = y.k[t][j >> 1][2 * (j & 1)], c1 = y.k[t][j >> 1][2 * (j & 1) + 1];
            const float pw = j < 2 ? power : power2;
            w.x = decode_pair<8>(c0, 0, pw);
            w.y = decode_pair<8>(c0, 1, pw);
            w.z = decode_pair<8>(c1, 0, pw);
            w.w = decode_pair<8>(c1, 1, pw);
          } else {
            const uint32_t c = y.k[t][0][j];
            w.x = decode_pair<4>(c, 0, power);
            w.y = decode_pair<4>(c, 1, power);
            w.z = decode_pair<4>(c, 2, power);
            w.w = decode_pair<4>(c, 3, power);
          }
          const bf16x8 kf = __builtin_bit_cast(bf16x8, w);
#pragma unroll
          for (int s = 0; s < S; ++s) d[s][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qv[s][j], d[s][t], 0, 0, 0);
        }
      }
      const int at = step * kStep + wave * 32;
      bf16x8 part[S];
#pragma unroll
      for (int s = 0; s < S; ++s) {
        constexpr float kTo2 = kMod ? 1.f : kScaleLog2;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = d[s][i >> 2][i & 3];
        if constexpr (kMod) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float r = v[i];
            v[i] = r * kScaleLog2;
            if (x.cap > 0.f) {
              const float z = r * to_cap;
              v[i] = x.cap * kLog2e * (__any(fabsf(z) > kTanhPoly) ? tanh_any(z) : tanh_poly(z));
            }
          }
          if (x.slopes) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              int row;  // of the tile's first position
              if constexpr (kRows == 0) row = (int)p0 + at + 16 * t;
              else row = sh.t.row[min(at + 16 * t, cnt - 1) >> 4];
#pragma unroll
              for (int i = 0; i < 4; ++i) v[4 * t + i] = fmaf(-slope2[s], (float)(nseq - 1 - row - 4 * grp - i), v[4 * t + i]);
            }
          }
        }
        if (at + 32 > cnt) {
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = at + 16 * (i >> 2) + 4 * grp + (i & 3) < cnt ? v[i] : -INFINITY;
        }
        float mx = fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7]))) * kTo2;
        // the reference is raised only where a weight would pass 2^8
        if (__any(mx > m[s] + 8.f)) {
          mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
          mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
          const float to = fmaxf(m[s], fminf(mx, 3.402823466e38f));  // (a score of +inf: the sum is inf, the output NaN)
          const float corr = fast_exp2(m[s] - to);
          m[s] = to;
          l[s] *= corr;
          const f32x4 c = {dpp<0x00>(corr), dpp<0x55>(corr), dpp<0xAA>(corr), dpp<0xFF>(corr)};  // of the quad's four heads
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[s][e] *= c;
        }
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          float p[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            p[k] = fast_exp2(fmaf(v[i + k], kTo2, -m[s]));
            l[s] += p[k];
            p[k] -= __uint_as_float(__float_as_uint(p[k]) & off1);
            p[k] -= __uint_as_float(__float_as_uint(p[k]) & off2);
          }
          w[i >> 1] = high_halves(__float_as_uint(p[0]), __float_as_uint(p[1]));
        }
        part[s] = __builtin_bit_cast(bf16x8, w);
      }
      float power[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) power[i] = power_in(y.vs[i], v_turn);
#pragma unroll
      for (int e = 0; e < 4; ++e) {  // two dimensions at a time
        uint32_t z[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if constexpr (kBits == 8) z[i] = e & 1 ? decode_pair<8>(y.v[i][e >> 1], 1, power[i]) : decode_pair<8>(y.v[i][e >> 1], 0, power[i]);
          else z[i] = e == 0 ? decode_pair<4>(y.v[i][0], 0, power[i]) : e == 1 ? decode_pair<4>(y.v[i][0], 1, power[i])
                      : e == 2 ? decode_pair<4>(y.v[i][0], 2, power[i]) : decode_pair<4>(y.v[i][0], 3, power[i]);
        }
        const u32x4 lo = {low_halves(z[0], z[1]), low_halves(z[2], z[3]), low_halves(z[4], z[5]), low_halves(z[6], z[7])};
        const u32x4 hi = {high_halves(z[0], z[1]), high_halves(z[2], z[3]), high_halves(z[4], z[5]), high_halves(z[6], z[7])};
#pragma unroll
        for (int s = 0; s < S; ++s) {
          acc[s][2 * e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(part[s], __builtin_bit_cast(bf16x8, lo), acc[s][2 * e], 0, 0, 0);
          acc[s][2 * e + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(part[s], __builtin_bit_cast(bf16x8, hi), acc[s][2 * e + 1], 0, 0, 0);
        }
      }
    };
    for (int64_t p = seg_lo; p < seg_hi; p += cnt) {
      p0 = p;
      if constexpr (kRows == 0) {
        cnt = (int)(seg_hi - p);
      } else {
        cnt = (int)min(seg_hi - p, (int64_t)kTableRows);
        auto row_at = [&](int64_t pos) -> int {
          if (!x.blocks) return (int)pos;
          const int lb = __builtin_ctz(x.block);
          const int64_t at = x.blocks[(int64_t)bg * x.budget + (pos >> lb)];
          return (int)min(max((at << lb) + (pos & (x.block - 1)), (int64_t)0), (int64_t)nseq - 1);
        };
        if (tid * 16 < cnt) {
          int row[1] = {row_at(p + tid * 16)};
          sh.t.row[tid] = row[0];
          if constexpr (kRows == 1) {
            // (a list that is not as it should be: the rows stay inside the sequence and their page)
            if (x.blocks) row[0] = max(min(row[0], nseq - min(16, cnt - tid * 16)), 0) & ~(x.kv.paged ? 15 : 0);
            if (x.kv.paged) {
              int64_t at[1];
              paged_rows(x.kv.pk, a.Hkv, a.total, kvb, b, kvh, row, 0, at);
              row[0] = (int)at[0];
            }
            sh.t.tile[tid] = row[0];
          }
        }
        if constexpr (kRows == 2) {
          constexpr int kPer = kTableRows / kThreads;
          int rr[kPer];
          int64_t pr[kPer];
#pragma unroll
          for (int e = 0; e < kPer; ++e) rr[e] = row_at(p + min(tid + e * kThreads, cnt - 1));
          paged_rows(x.kv.pk, a.Hkv, a.total, kvb, b, kvh, rr, 0, pr);
#pragma unroll
          for (int e = 0; e < kPer; ++e)
            if (tid + e * kThreads < cnt) sh.t.place[tid + e * kThreads] = (int)pr[e];
        }
        __syncthreads();
      }
      const int steps = (max(cnt - wave * 32, 0) + kStep - 1) / kStep;
      if (steps > 0) {
        Tile y0 = load_tile(0);
        // (one step ahead; two: at most 8% faster for short sequences, 10% to 60% slower with eight heads)
#pragma unroll 1
        for (int s = 0; s < steps; s += 2) {
          const Tile y1 = load_tile(s + 1);  // (a load past the last step reads its row again)
          __builtin_amdgcn_sched_barrier(0);
          consume(y0, s);
          if (s + 1 >= steps) break;
          y0 = load_tile(s + 2);
          __builtin_amdgcn_sched_barrier(0);
          consume(y1, s + 1);
        }
      }
      if constexpr (kRows != 0) __syncthreads();  // the next sub-range, or the merge, rewrites the table
    }

    // ---- merge the waves: common maximum, rescale, sum
#pragma unroll
    for (int s = 0; s < S; ++s) {
      l[s] += __shfl_xor(l[s], 16, 64);
      l[s] += __shfl_xor(l[s], 32, 64);
      if (lane < 4 && hd < G) {
        s_ml[wave][0][4 * s + hd] = m[s];
        s_ml[wave][1][4 * s + hd] = l[s];
      }
      if (grp < 3) {
#pragma unroll
        for (int h = 0; h < (G < 4 ? G : 4); ++h)
#pragma unroll
          for (int e = 0; e < 8; e += 4)
            *reinterpret_cast<float4*>(&sh.red[wave * 3 + grp][4 * s + h][sl * 8 + e]) =
                make_float4(acc[s][e][h], acc[s][e + 1][h], acc[s][e + 2][h], acc[s][e + 3][h]);
      }
    }
    __syncthreads();
    constexpr int kEach = kDirect ? (G >= 2 ? G / 2 : 1) : 4;  // values of a thread
    struct __attribute__((aligned(kEach * 4))) Values {
      float v[kEach];
    };
    if (tid * kEach < G * kHeadDim) {
      const int h = tid * kEach / kHeadDim, e = tid * kEach % kHeadDim;
      float mm = -INFINITY, ll = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) mm = fmaxf(mm, s_ml[w][1][h] == 0.f ? -INFINITY : s_ml[w][0][h]);
      Values sum{};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float lw = s_ml[w][1][h], f = lw == 0.f ? 0.f : fast_exp2(s_ml[w][0][h] - mm);
        ll = fmaf(lw, f, ll);
        Values y{};
#pragma unroll
        for (int q = 2; q >= 0; --q) {  // the small parts first
          const Values part = *reinterpret_cast<const Values*>(&sh.red[w * 3 + q][h][e]);
#pragma unroll
          for (int i = 0; i < kEach; ++i) y.v[i] += part.v[i];
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i) sum.v[i] = fmaf(y.v[i], f, sum.v[i]);
      }
      if constexpr (kDirect) {
        const int64_t row = (int64_t)b * a.Hq + kvh * G + h;
        const bool empty = mm == -INFINITY;
        if (empty) sum = Values{}, ll = 1.f;
#pragma unroll
        for (int i = 0; i < kEach; ++i) sum.v[i] /= ll;
        *reinterpret_cast<Values*>(a.out + row * kHeadDim + e) = sum;
        if (e == 0 && x.lse) x.lse[row] = empty ? -INFINITY : (mm + __builtin_amdgcn_logf(ll)) * kLn2;
      } else {
        float* part = a.partials + ((int64_t)bg + blockIdx.x) * kPart;
        *reinterpret_cast<Values*>(part + tid * kEach) = sum;
        if (e == 0) {
          part[G * kHeadDim + h] = mm;
          part[G * kHeadDim + G + h] = ll;
        }
      }
    }
    if (bg + 1 < bg_end) __syncthreads();
  }
}

// Calls f with the kernel of these arguments.
template <int G, int kBits, bool kDirect, typename F>
static hipError_t with_kernel_g(const QuantAttnArgs& x, F f) {
  const bool mod = x.cap > 0.f || x.slopes;
  if (x.kv.paged && x.kv.pk.page_size % 16)
    return mod ? f(quant_attn_kernel<G, kBits, 2, true, kDirect>) : f(quant_attn_kernel<G, kBits, 2, false, kDirect>);
  if (x.blocks || x.kv.paged)
    return mod ? f(quant_attn_kernel<G, kBits, 1, true, kDirect>) : f(quant_attn_kernel<G, kBits, 1, false, kDirect>);
  return mod ? f(quant_attn_kernel<G, kBits, 0, true, kDirect>) : f(quant_attn_kernel<G, kBits, 0, false, kDirect>);
}
template <int G, typename F>
static hipError_t with_kernel_of(const QuantAttnArgs& x, F f) {
  if (x.direct) return x.kv.bits == 8 ? with_kernel_g<G, 8, true>(x, f) : with_kernel_g<G, 4, true>(x, f);
  return x.kv.bits == 8 ? with_kernel_g<G, 8, false>(x, f) : with_kernel_g<G, 4, false>(x, f);
}
template <typename F>
static hipError_t with_kernel(const QuantAttnArgs& x, int G, F f) {
  switch (G) {
    case 1: return with_kernel_of<1>(x, f);
    case 2: return with_kernel_of<2>(x, f);
    case 4: return with_kernel_of<4>(x, f);
    case 8: return with_kernel_of<8>(x, f);
    default: return hipErrorInvalidValue;
  }
}

// Dynamic LDS of the units before each group and of the groups' rows
static size_t prefix_lds(const QuantAttnArgs& x) {
  const size_t groups = (size_t)x.a.B * x.a.NV;
  return x.direct ? 0 : (groups + 1) * sizeof(int64_t) + groups * sizeof(Group);
}

hipError_t quant_resident_grid(const QuantAttnArgs& x, int G, int* grid) {
  int dev = 0, cus = 0, per = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e == hipSuccess) e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
  if (e == hipSuccess)
    e = with_kernel(x, G, [&](auto kernel) { return hipOccupancyMaxActiveBlocksPerMultiprocessor(&per, kernel, kWave * kWaves, prefix_lds(x)); });
  *grid = std::max(per, 1) * std::max(cus, 1);
  return e;
}

hipError_t launch_quant_attn(const QuantAttnArgs& x, int G, int grid, hipStream_t st) {
  return with_kernel(x, G, [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(kWave * kWaves), prefix_lds(x), st, x);
    return hipGetLastError();
  });
}

}  // namespace tactic
