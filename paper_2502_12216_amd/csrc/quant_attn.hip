// One new token per sequence over a quantised cache: all of its rows or those of chosen
// blocks, split over the workgroups and joined by the combine of the dense decode.
//
// A row of K and V is 264 or 136 bytes for 512 G operations: bound by HBM as long as
// codes become products in few instructions.  A wave takes 32 rows a step, and
// everything stays in the lanes that loaded it:
//  - Scores: two tiles of 16 rows, each four v_mfma_f32_16x16x32_bf16 with the rows of K as
//    the first operand - lane l has row l % 16, dimensions 32 (l / 16) .. + 31, which is one
//    group and one power, converted to bf16 exactly - and four query heads as the columns,
//    repeated four times.  So lane l receives the scores of head l % 4 for the rows
//    4 (l / 16) .. + 3 of either tile, exactly once for each lane that needs them.
//  - Values: lanes with l % 16 < 8 take the first tile, the others the second: rows
//    4 (l / 16) .. + 3 of it, 16 dimensions each, so that a quad of lanes has the weights of
//    four heads and the values of four dimensions of the same four rows: one block of
//    v_mfma_f32_4x4x4_16b_bf16 for each of the lane's dimensions, with the weights split
//    into three bf16 parts whose sum is exact.
// (The instructions that multiply 8 and 4 bit codes themselves add with fewer bits: 9e-5
// of the absolute sum for a row of 128 codes, where fp32 has 6e-8.)
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
constexpr int64_t kQuantShare = 256;  // rows of the least share
constexpr int kTableRows = 2048;      // rows looked up at once

typedef short bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
__device__ __forceinline__ bf16x4 four(uint32_t lo, uint32_t hi) {
  u32x2 w;
  w.x = lo;
  w.y = hi;
  return __builtin_bit_cast(bf16x4, w);
}

// Four fp32 weights as three bf16 operands whose sum is exact: the upper 8 bits of the
// significand, the next 8 of the rest, the rest
__device__ __forceinline__ void three_parts(const float (&p)[4], bf16x4 (&part)[3]) {
  uint32_t h[4], m[4], r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    h[i] = __float_as_uint(p[i]);
    const float x = p[i] - __uint_as_float(h[i] & 0xffff0000u);
    m[i] = __float_as_uint(x);
    r[i] = __float_as_uint(x - __uint_as_float(m[i] & 0xffff0000u));
  }
  part[0] = four(high_halves(h[0], h[1]), high_halves(h[2], h[3]));
  part[1] = four(high_halves(m[0], m[1]), high_halves(m[2], m[3]));
  part[2] = four(high_halves(r[0], r[1]), high_halves(r[2], r[3]));
}

// Rows that group bg attends: its sequence's, or those of its chosen blocks (ascending, so
// that only the last one may be the sequence's last, of fewer rows).
__device__ __forceinline__ int64_t rows_of(const QuantAttnArgs& x, int bg) {
  const int b = bg / x.a.NV;
  const int64_t n = seq_tokens(x.a.kv_indptr, x.a.seq_len, b);
  if (!x.blocks) return n;
  const int count = min(max(x.counts[bg], 0), x.budget);
  if (count == 0 || n == 0) return 0;
  const int lb = __builtin_ctz(x.block);
  const int64_t last = x.blocks[(int64_t)bg * x.budget + count - 1];
  return ((int64_t)(count - 1) << lb) + min(max(n - (last << lb), (int64_t)1), (int64_t)x.block);
}

// kTable: rows are looked up (pages or chosen blocks), else they are the positions
template <int G, int kBits, bool kTable, bool kMod>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(G == 8 ? 1 : 2)))
void quant_attn_kernel(QuantAttnArgs x) {
  constexpr int kPart = G * (kHeadDim + 2);
  constexpr int S = G == 8 ? 2 : 1;         // sets of four heads
  constexpr int RB = kRowBytes<kBits>;
  constexpr int KW = kBits == 8 ? 2 : 1;    // 16-byte words of a lane's group of K
  constexpr int VW = kBits == 8 ? 4 : 2;    // 4-byte words of a lane's 16 values
  constexpr int kAhead = kBits == 8 ? 1 : 2;  // steps loaded ahead
  const AttnArgs& a = x.a;
  extern __shared__ int64_t s_prefix[];     // [B * NV + 1] units before each group
  union Shared {
    struct {
      int place[kTableRows];                // row in the arrays, from the head's (spans) or their start (pages)
      int row[kMod ? kTableRows : 1];       // row of the sequence
    } t;
    float red[16][G][kHeadDim];             // the merge: four row groups of four waves
  };
  __shared__ __align__(16) Shared sh;
  __shared__ float s_ml[32][2][G];
  __shared__ float s_M[G], s_L[G];
  __shared__ int64_t s_wsum[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int sl = lane & 15, grp = lane >> 4, half = sl >> 3, hd = sl & 3;
  const int BG = a.B * a.NV;
  auto units = [&](int bg) { const int64_t n = rows_of(x, bg); return n > 0 ? n + kSegmentCost : 0; };
  {
    const int per = (BG + 255) / 256, g0 = min(BG, tid * per), g1 = min(BG, g0 + per);
    const int64_t u_first = g0 < g1 ? units(g0) : 0;
    int64_t loc = u_first;
    for (int bg = g0 + 1; bg < g1; ++bg) loc += units(bg);
    const int64_t incl = wave_incl_scan(loc);
    if (lane == kWave - 1) s_wsum[wave] = incl;
    __syncthreads();
    int64_t run = incl - loc;
    for (int w = 0; w < wave; ++w) run += s_wsum[w];
    for (int bg = g0; bg < g1; ++bg) {
      s_prefix[bg] = run;
      run += bg == g0 ? u_first : units(bg);
    }
    if (tid == 255) s_prefix[BG] = run;
    __syncthreads();
  }
  const int64_t total = s_prefix[BG];
  const int64_t share = max((total + gridDim.x - 1) / gridDim.x, kQuantShare);
  if (blockIdx.x == 0) {  // for the combine
    if (tid == 0) a.ameta[0] = share;
    for (int bg = tid; bg <= BG; bg += 256) a.ameta[1 + bg] = s_prefix[bg];
  }
  const int64_t t0 = (int64_t)blockIdx.x * share, t1 = min(total, t0 + share);
  if (t0 >= t1) return;
  int bg0 = 0, bgh = BG - 1;  // the largest group that starts at or before t0
  while (bg0 < bgh) {
    const int mid = (bg0 + bgh + 1) >> 1;
    if (s_prefix[mid] <= t0) bg0 = mid;
    else bgh = mid - 1;
  }
  bg0 = __builtin_amdgcn_readfirstlane(bg0);

  for (int bg = bg0; bg < BG && s_prefix[bg] < t1; ++bg) {
    const int64_t first = s_prefix[bg] + kSegmentCost;
    const int64_t seg_lo = max(t0, first) - first, seg_hi = min(t1, s_prefix[bg + 1]) - first;
    if (seg_lo >= seg_hi) continue;
    const int b = bg / a.NV, kvh = bg % a.NV;
    const int64_t kvb = a.kv_indptr[b];
    const int nseq = (int)seq_tokens(a.kv_indptr, a.seq_len, b);

    // the queries: dimensions 32 grp .. + 31 of head hd of each set
    bf16x8 qv[S][4];
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const uint16_t* qp = a.q + ((int64_t)b * a.Hq + kvh * G + (G >= 4 ? 4 * s + hd : hd % G)) * kHeadDim + grp * 32;
#pragma unroll
      for (int j = 0; j < 4; ++j) qv[s][j] = *reinterpret_cast<const bf16x8*>(qp + 8 * j);
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
    // reference maximum and sum of this lane's heads over its rows; sums of values, a
    // vector of four heads for each of the lane's 16 dimensions
    float m[S], l[S];
    f32x4 acc[S][16];
#pragma unroll
    for (int s = 0; s < S; ++s) {
      m[s] = -INFINITY;
      l[s] = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[s][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int64_t base = x.kv.paged ? 0 : (int64_t)kvh * a.total + kvb;
    const uint8_t* Kb = x.kv.K + base * RB + grp * (RB / 4);
    const uint8_t* Ks = x.kv.K_scale + base * 4 + grp;
    const uint8_t* Vb = x.kv.V + base * RB + (sl & 7) * (RB / 8);
    const uint8_t* Vs = x.kv.V_scale + base * 4 + ((sl & 7) >> 1);
    int cnt = 0;
    int64_t p0 = 0;
    struct Tile {
      u32x4 k[2][KW];
      uint32_t v[4][VW];
      uint8_t ks[2], vs[4];
    };
    // step `step` of this wave: positions 128 step + 32 wave .. + 31 of the sub-range; those
    // past its end read its last row, which the group attends anyway
    auto load_tile = [&](int step) __attribute__((always_inline)) -> Tile {
      Tile r;
      const int at = step * 128 + wave * 32;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int pos = min(at + 16 * t + sl, cnt - 1);
        const int64_t row = kTable ? (int64_t)sh.t.place[pos] : p0 + pos;
        const uint8_t* p = Kb + row * RB;
#pragma unroll
        for (int w = 0; w < KW; ++w) r.k[t][w] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p) + w);
        r.ks[t] = Ks[row * 4];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int pos = min(at + 16 * half + 4 * grp + i, cnt - 1);
        const int64_t row = kTable ? (int64_t)sh.t.place[pos] : p0 + pos;
        const uint8_t* p = Vb + row * RB;
        if constexpr (kBits == 8) {
          const u32x4 w = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
          r.v[i][0] = w.x; r.v[i][1] = w.y; r.v[i][2] = w.z; r.v[i][3] = w.w;
        } else {
          const u32x2 w = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p));
          r.v[i][0] = w.x; r.v[i][1] = w.y;
        }
        r.vs[i] = Vs[row * 4];
      }
      return r;
    };
    auto consume = [&](const Tile& y, int step) __attribute__((always_inline)) {
      f32x4 d[S][2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const float power = power_of(y.ks[t]);
#pragma unroll
        for (int s = 0; s < S; ++s) d[s][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          u32x4 w;
          if constexpr (kBits == 8) {
            const uint32_t c0 = y.k[t][j >> 1][2 * (j & 1)], c1 = y.k[t][j >> 1][2 * (j & 1) + 1];
            w.x = decode_pair<8>(c0, 0, power);
            w.y = decode_pair<8>(c0, 1, power);
            w.z = decode_pair<8>(c1, 0, power);
            w.w = decode_pair<8>(c1, 1, power);
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
      const int pos0 = step * 128 + wave * 32 + 16 * half + 4 * grp;
      const bool whole = step * 128 + wave * 32 + 32 <= cnt;
      bf16x4 part[S][3];
#pragma unroll
      for (int s = 0; s < S; ++s) {
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float r = half ? d[s][1][i] : d[s][0][i];
          v[i] = r * kScaleLog2;
          if constexpr (kMod) {
            if (x.cap > 0.f) {
              const float z = r * to_cap;
              v[i] = x.cap * kLog2e * (__any(fabsf(z) > kTanhPoly) ? tanh_any(z) : tanh_poly(z));
            }
            if (x.slopes) {
              const int pos = min(pos0 + i, cnt - 1);
              const int row = kTable ? sh.t.row[pos] : (int)(p0 + pos);
              v[i] = fmaf(-slope2[s], (float)(nseq - 1 - row), v[i]);
            }
          }
        }
        if (!whole) {
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = pos0 + i < cnt ? v[i] : -INFINITY;
        }
        // the reference is raised only where a weight would pass 2^8
        float mn = fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]));
        mn = fminf(mn, 3.402823466e38f);  // a score of +inf: the sum is inf, the output NaN
        if (__any(mn > m[s] + 8.f)) {
          const float to = fmaxf(m[s], mn);
          const float corr = to > m[s] ? fast_exp2(m[s] - to) : 1.f;
          m[s] = to;
          l[s] *= corr;
          const f32x4 c = {dpp<0x00>(corr), dpp<0x55>(corr), dpp<0xAA>(corr), dpp<0xFF>(corr)};  // of the quad's four heads
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[s][e] *= c;
        }
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[i] = v[i] == -INFINITY ? 0.f : fast_exp2(v[i] - m[s]);
          l[s] += p[i];
        }
        three_parts(p, part[s]);
      }
      // the values, eight dimensions at a time
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        bf16x4 vt[8];
#pragma unroll
        for (int w = 0; w < 4; ++w) {  // pairs 4 c + w of the 8
          uint32_t z[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float power = power_of(y.vs[i]);
            if constexpr (kBits == 8) z[i] = w & 1 ? decode_pair<8>(y.v[i][2 * c + (w >> 1)], 1, power) : decode_pair<8>(y.v[i][2 * c + (w >> 1)], 0, power);
            else z[i] = w == 0 ? decode_pair<4>(y.v[i][c], 0, power) : w == 1 ? decode_pair<4>(y.v[i][c], 1, power)
                        : w == 2 ? decode_pair<4>(y.v[i][c], 2, power) : decode_pair<4>(y.v[i][c], 3, power);
          }
          vt[2 * w] = four(low_halves(z[0], z[1]), low_halves(z[2], z[3]));
          vt[2 * w + 1] = four(high_halves(z[0], z[1]), high_halves(z[2], z[3]));
        }
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
          for (int k = 2; k >= 0; --k)
#pragma unroll
            for (int e = 0; e < 8; ++e)
              acc[s][8 * c + e] = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(part[s][k], vt[e], acc[s][8 * c + e], 0, 0, 0);
      }
    };
    for (int64_t p = seg_lo; p < seg_hi; p += cnt) {
      p0 = p;
      if constexpr (!kTable) {
        cnt = (int)(seg_hi - p);
      } else {
        cnt = (int)min(seg_hi - p, (int64_t)kTableRows);
        constexpr int kPer = kTableRows / 256;
        int rr[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          const int64_t pos = p + min(tid + e * 256, cnt - 1);
          if (x.blocks) {
            const int lb = __builtin_ctz(x.block);
            const int64_t at = x.blocks[(int64_t)bg * x.budget + (pos >> lb)];
            rr[e] = (int)min(max((at << lb) + (pos & (x.block - 1)), (int64_t)0), (int64_t)nseq - 1);
          } else {
            rr[e] = (int)pos;
          }
        }
        if constexpr (kMod) {
#pragma unroll
          for (int e = 0; e < kPer; ++e)
            if (tid + e * 256 < cnt) sh.t.row[tid + e * 256] = rr[e];
        }
        if (x.kv.paged) {
          int64_t pr[kPer];
          paged_rows(x.kv.pk, a.Hkv, a.total, kvb, b, kvh, rr, 0, pr);
#pragma unroll
          for (int e = 0; e < kPer; ++e) rr[e] = (int)pr[e];
        }
#pragma unroll
        for (int e = 0; e < kPer; ++e)
          if (tid + e * 256 < cnt) sh.t.place[tid + e * 256] = rr[e];
        __syncthreads();
      }
      const int steps = (max(cnt - wave * 32, 0) + 127) / 128;
      if (steps > 0) {
        Tile y0 = load_tile(0);
        if constexpr (kAhead == 1) {
#pragma unroll 1
          for (int s = 0; s < steps; s += 2) {
            const Tile y1 = load_tile(s + 1);
            consume(y0, s);
            if (s + 1 >= steps) break;
            y0 = load_tile(s + 2);
            consume(y1, s + 1);
          }
        } else {
          Tile y1 = load_tile(1);
#pragma unroll 1
          for (int s = 0; s < steps; s += 3) {
            Tile y2 = load_tile(s + 2);
            consume(y0, s);
            if (s + 1 >= steps) break;
            y0 = load_tile(s + 3);
            consume(y1, s + 1);
            if (s + 2 >= steps) break;
            y1 = load_tile(s + 4);
            consume(y2, s + 2);
          }
        }
      }
      if constexpr (kTable) __syncthreads();  // the next sub-range, or the merge, rewrites the table
    }

    // ---- merge: 32 states of every head (wave, row group, half): common maximum, rescale, sum
    const int state = wave * 8 + grp * 2 + half;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      if (m[s] == -INFINITY && l[s] != l[s]) m[s] = 0.f;  // (a maximum passes NaN over: where no other score was there the sum says that some was)
      if ((sl & 7) < 4 && hd < G) {
        s_ml[state][0][4 * s + hd] = m[s];
        s_ml[state][1][4 * s + hd] = l[s];
      }
    }
    __syncthreads();
    if (tid < G) {
      float mm = -INFINITY;
      for (int q = 0; q < 32; ++q) mm = fmaxf(mm, s_ml[q][0][tid]);
      float ll = 0.f;
      for (int q = 0; q < 32; ++q) {
        const float mq = s_ml[q][0][tid];
        ll += mq == -INFINITY ? 0.f : s_ml[q][1][tid] * fast_exp2(mq - mm);
      }
      s_M[tid] = mm;
      s_L[tid] = ll;
    }
    __syncthreads();
    float* part = a.partials + ((int64_t)bg + blockIdx.x) * kPart;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const float sc = m[s] == -INFINITY ? 0.f : fast_exp2(m[s] - s_M[G >= 4 ? 4 * s + hd : hd % G]);
      const f32x4 c = {dpp<0x00>(sc), dpp<0x55>(sc), dpp<0xAA>(sc), dpp<0xFF>(sc)};
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        f32x4 y = acc[s][e] * c;
#pragma unroll
        for (int h = 0; h < (G < 4 ? G : 4); ++h) {
          const float z = y[h] + dpp<0x128>(y[h]);  // row_ror:8, the other half's rows
          acc[s][e][h] = z;
        }
      }
      if (half == 0) {
#pragma unroll
        for (int h = 0; h < (G < 4 ? G : 4); ++h)
#pragma unroll
          for (int e = 0; e < 16; e += 4)
            *reinterpret_cast<float4*>(&sh.red[wave * 4 + grp][4 * s + h][(sl & 7) * 16 + e]) =
                make_float4(acc[s][e][h], acc[s][e + 1][h], acc[s][e + 2][h], acc[s][e + 3][h]);
      }
    }
    __syncthreads();
    if (tid * 4 < G * kHeadDim) {
      const int h = tid * 4 / kHeadDim, e = tid * 4 % kHeadDim;
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int q = 0; q < 16; ++q) {
        const float4 v = *reinterpret_cast<const float4*>(&sh.red[q][h][e]);
        sum.x += v.x;
        sum.y += v.y;
        sum.z += v.z;
        sum.w += v.w;
      }
      *reinterpret_cast<float4*>(part + tid * 4) = sum;
    }
    if (tid < G) {
      part[G * kHeadDim + tid] = s_M[tid];
      part[G * kHeadDim + G + tid] = s_L[tid];
    }
    __syncthreads();
  }
}

// Calls f with the kernel of these arguments.
template <int G, int kBits, typename F>
static hipError_t with_kernel_g(const QuantAttnArgs& x, F f) {
  const bool table = x.blocks || x.kv.paged, mod = x.cap > 0.f || x.slopes;
  if (table) return mod ? f(quant_attn_kernel<G, kBits, true, true>) : f(quant_attn_kernel<G, kBits, true, false>);
  return mod ? f(quant_attn_kernel<G, kBits, false, true>) : f(quant_attn_kernel<G, kBits, false, false>);
}
template <typename F>
static hipError_t with_kernel(const QuantAttnArgs& x, int G, F f) {
  const bool eight = x.kv.bits == 8;
  switch (G) {
    case 1: return eight ? with_kernel_g<1, 8>(x, f) : with_kernel_g<1, 4>(x, f);
    case 2: return eight ? with_kernel_g<2, 8>(x, f) : with_kernel_g<2, 4>(x, f);
    case 4: return eight ? with_kernel_g<4, 8>(x, f) : with_kernel_g<4, 4>(x, f);
    case 8: return eight ? with_kernel_g<8, 8>(x, f) : with_kernel_g<8, 4>(x, f);
    default: return hipErrorInvalidValue;
  }
}

hipError_t quant_resident_grid(const QuantAttnArgs& x, int G, int* grid) {
  int dev = 0, cus = 0, per = 0;
  const size_t lds = ((size_t)x.a.B * x.a.NV + 1) * sizeof(int64_t);
  hipError_t e = hipGetDevice(&dev);
  if (e == hipSuccess) e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
  if (e == hipSuccess)
    e = with_kernel(x, G, [&](auto kernel) { return hipOccupancyMaxActiveBlocksPerMultiprocessor(&per, kernel, 256, lds); });
  *grid = std::max(per, 1) * std::max(cus, 1);
  return e;
}

hipError_t launch_quant_attn(const QuantAttnArgs& x, int G, int grid, hipStream_t st) {
  const size_t lds = ((size_t)x.a.B * x.a.NV + 1) * sizeof(int64_t);
  return with_kernel(x, G, [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), lds, st, x);
    return hipGetLastError();
  });
}

}  // namespace tactic
