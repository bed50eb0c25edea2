// Blocks of a cache that a token may look at most, by a cheap score.
//
// The score of block j for query head h is the largest product that a key inside the
// block's bounds could have with the query, u_hj = sum_d (q_d >= 0 ? q_d hi_jd : q_d lo_jd).
// A group's score of a block is the best of its heads', each counted from that head's
// best block: max_h (u_hj - max_i u_hi).  The products of two bf16 are exact and their
// sums are in 64 bits, so that the order of blocks does not depend on how they are summed.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "common.hpp"
#include "kernels.hpp"
#include "quant.hpp"

namespace tactic {

// 64 blocks of one KV head for its G query heads, four heads at a time (their queries are 128
// registers).  A block is 512 bytes and 2 G 128 fused operations in 64 bits.
template <int G>
__global__ __launch_bounds__(256) void block_score_kernel(SelectArgs a) {
  constexpr int H = G < 4 ? G : 4;
  __shared__ double s_top[16][G];
  const int tid = threadIdx.x, sl = tid & 15, sub = tid >> 4;
  const int g = blockIdx.y, b = blockIdx.z;
  const int lb = __builtin_ctz(a.block);
  const int64_t kvb = a.kv_indptr[b], n = seq_tokens(a.kv_indptr, a.seq_len, b);
  const int64_t nb = (n + a.block - 1) >> lb;
  const int64_t j0 = (int64_t)blockIdx.x * kSelectRows;
  if (j0 >= nb || nb <= a.budget) return;  // (all of them are chosen)
  const uint16_t* bounds = a.bounds + ((int64_t)g * ((a.total >> lb) + a.B) + first_block(kvb, lb, b)) * (2 * kHeadDim) + sl * 8;
  uint4 lo[4], hi[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t j = min(j0 + 16 * i + sub, nb - 1);
    lo[i] = load_stream16(bounds + j * (2 * kHeadDim));
    hi[i] = load_stream16(bounds + j * (2 * kHeadDim) + kHeadDim);
  }
#pragma unroll 1
  for (int h0 = 0; h0 < G; h0 += H) {
    const int64_t head = (int64_t)b * a.Hq + g * G + h0;
    double pos[H][8], neg[H][8], best[H];
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const uint4 w = *reinterpret_cast<const uint4*>(a.q + (head + h) * kHeadDim + sl * 8);
      const uint32_t u[4] = {w.x, w.y, w.z, w.w};
      best[h] = -INFINITY;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float q = e & 1 ? bf16hi(u[e >> 1]) : bf16lo(u[e >> 1]);
        pos[h][e] = q < 0.f ? 0.0 : (double)q;
        neg[h][e] = q < 0.f ? (double)q : 0.0;
      }
    }
    double* scores = a.scores + head * a.max_blocks;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t j = j0 + 16 * i + sub;
      double u[H];
#pragma unroll
      for (int h = 0; h < H; ++h) u[h] = 0.0;
      const uint32_t l[4] = {lo[i].x, lo[i].y, lo[i].z, lo[i].w}, t[4] = {hi[i].x, hi[i].y, hi[i].z, hi[i].w};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double x = (double)(e & 1 ? bf16hi(l[e >> 1]) : bf16lo(l[e >> 1]));
        const double y = (double)(e & 1 ? bf16hi(t[e >> 1]) : bf16lo(t[e >> 1]));
#pragma unroll
        for (int h = 0; h < H; ++h) u[h] = fma(neg[h][e], x, fma(pos[h][e], y, u[h]));
      }
#pragma unroll
      for (int h = 0; h < H; ++h) {
        u[h] = sum16d(u[h]);
        if (j < nb) {
          best[h] = fmax(best[h], u[h]);  // (NaN is passed over)
          if (sl == 0) scores[(int64_t)h * a.max_blocks + j] = u[h];
        }
      }
    }
    if (sl == 0) {
#pragma unroll
      for (int h = 0; h < H; ++h) s_top[sub][h0 + h] = best[h];
    }
  }
  __syncthreads();
  if (tid < G) {
    double v = s_top[0][tid];
    for (int i = 1; i < 16; ++i) v = fmax(v, s_top[i][tid]);
    a.top[((int64_t)b * a.Hq + g * G + tid) * a.tops + blockIdx.x] = v;
  }
}

// Scores as integers that order as they do, NaN as +inf
__device__ __forceinline__ uint64_t order_key(double x) {
  if (x != x) x = INFINITY;
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  return u >> 63 ? ~u : u | 0x8000000000000000ull;
}

// The `budget` blocks of the largest keys of one KV head, ascending.  A radix selection:
// digits of 11 bits from the first bit in which the keys differ (so that a digit spreads over
// the scores there are), each with a histogram in LDS of the keys still level; it ends
// as soon as all keys of the digit that holds the last one are wanted.  Thread t has blocks t kPer ..,
// so that ranks and places are one scan; kPer = 0: the keys lie in the workspace.
template <int kPer>
__global__ __launch_bounds__(1024) void block_select_kernel(SelectArgs a) {
  constexpr int kBins = 2048, kThreads = 1024;
  __shared__ uint32_t s_hist[kBins];
  __shared__ double s_best[8];
  __shared__ uint64_t s_min[16], s_max[16];
  __shared__ uint32_t s_wave[16][2];
  __shared__ uint32_t s_digit, s_above, s_in;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int g = blockIdx.x, b = blockIdx.y;
  const int lb = __builtin_ctz(a.block), G = a.G;
  const int64_t n = seq_tokens(a.kv_indptr, a.seq_len, b);
  const int nb = (int)((n + a.block - 1) >> lb), want = min(a.budget, nb);
  int32_t* out = a.blocks + ((int64_t)b * a.Hkv + g) * a.budget;
  if (tid == 0) a.counts[(int64_t)b * a.Hkv + g] = want;
  for (int i = want + tid; i < a.budget; i += kThreads) out[i] = -1;
  if (nb <= a.budget) {
    for (int i = tid; i < want; i += kThreads) out[i] = i;
    return;
  }
  // every head's best score: a wave for each
  if (wave < G) {
    const double* top = a.top + ((int64_t)b * a.Hq + g * G + wave) * a.tops;
    double v = -INFINITY;
    for (int i = lane; i < (nb + kSelectRows - 1) / kSelectRows; i += kWave) v = fmax(v, top[i]);
    v = wave_allmax_d(v);
    if (lane == 0) s_best[wave] = v;
  }
  __syncthreads();
  const double* scores = a.scores + ((int64_t)b * a.Hq + g * G) * a.max_blocks;
  uint64_t* stored = a.keys + ((int64_t)b * a.Hkv + g) * a.max_blocks;
  const int per = kPer ? kPer : (nb + kThreads - 1) / kThreads;
  const int j0 = tid * per;
  auto key_of = [&](int j) -> uint64_t {
    if (j < a.first || j >= nb - a.last) return ~0ull;
    double best = -INFINITY;
    bool odd = false;
    for (int h = 0; h < G; ++h) {
      const double d = scores[(int64_t)h * a.max_blocks + j] - s_best[h];
      odd |= d != d;
      best = fmax(best, d);
    }
    return order_key(odd ? INFINITY : best);
  };
  uint64_t held[kPer ? kPer : 1];
  uint64_t least = ~0ull, most = 0;
  if constexpr (kPer > 0) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int j = j0 + i;
      held[i] = j < nb ? key_of(j) : 0;
      if (j < nb) {
        least = min(least, held[i]);
        most = max(most, held[i]);
      }
    }
  } else {
    for (int j = tid; j < nb; j += kThreads) {  // (written and read by the same workgroup only)
      const uint64_t k = key_of(j);
      stored[j] = k;
      least = min(least, k);
      most = max(most, k);
    }
    __threadfence_block();
    __syncthreads();
  }
  auto each = [&](auto f) __attribute__((always_inline)) {  // (block, key) of this thread's blocks in order
    if constexpr (kPer > 0) {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (j0 + i < nb) f(j0 + i, held[i]);
    } else {
      for (int j = j0; j < min(nb, j0 + per); ++j) f(j, stored[j]);
    }
  };
  for (int d = 32; d >= 1; d /= 2) {
    least = min(least, (uint64_t)__shfl_xor((unsigned long long)least, d, 64));
    most = max(most, (uint64_t)__shfl_xor((unsigned long long)most, d, 64));
  }
  if (lane == 0) {
    s_min[wave] = least;
    s_max[wave] = most;
  }
  __syncthreads();
  for (int w = 0; w < 16; ++w) {
    least = min(least, s_min[w]);
    most = max(most, s_max[w]);
  }
  // keys agree above bit `low` with `prefix`; of those `need` are wanted
  int low = least == most ? 0 : 64 - __clzll((long long)(least ^ most));
  uint64_t prefix = low >= 64 ? 0 : most >> low;
  uint32_t need = (uint32_t)want;
  bool all = least == most ? (uint32_t)nb == need : false;
  auto level = [&](uint64_t k) { return low >= 64 || k >> low == prefix; };
  while (!all && low > 0) {
    const int bits = min(low, 11), shift = low - bits;
    for (int i = tid; i < kBins; i += kThreads) s_hist[i] = 0;
    __syncthreads();
    each([&](int, uint64_t k) {
      if (level(k)) atomicAdd(&s_hist[(k >> shift) & ((1u << bits) - 1)], 1u);
    });
    __syncthreads();
    // thread t: bins 2 t and 2 t + 1 counted from the top
    const uint32_t c0 = s_hist[kBins - 1 - 2 * tid], c1 = s_hist[kBins - 2 - 2 * tid];
    const uint32_t incl = wave_incl_scan(c0 + c1);
    if (lane == 63) s_wave[wave][0] = incl;
    __syncthreads();
    uint32_t ahead = incl - c0 - c1;
    for (int w = 0; w < wave; ++w) ahead += s_wave[w][0];
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
    prefix = low >= 64 ? (uint64_t)s_digit : prefix << bits | s_digit;
    need -= s_above;
    all = s_in == need;
    low = shift;
  }
  // chosen: keys above the prefix, and of those level with it all or the first `need`
  uint32_t above = 0, same = 0;
  each([&](int, uint64_t k) {
    const uint64_t p = low >= 64 ? 0 : k >> low;
    above += p > prefix;
    same += p == prefix;
  });
  const uint32_t ia = wave_incl_scan(above), is = wave_incl_scan(same);
  if (lane == 63) {
    s_wave[wave][0] = ia;
    s_wave[wave][1] = is;
  }
  __syncthreads();
  uint32_t pa = ia - above, ps = is - same;
  for (int w = 0; w < wave; ++w) {
    pa += s_wave[w][0];
    ps += s_wave[w][1];
  }
  each([&](int j, uint64_t k) {
    const uint64_t p = low >= 64 ? 0 : k >> low;
    const bool level_here = p == prefix, take = p > prefix || (level_here && ps < need);
    if (take) out[pa + min(ps, need)] = j;
    pa += p > prefix;
    ps += level_here;
  });
}

hipError_t launch_block_scores(const SelectArgs& a, hipStream_t st) {
  const dim3 grid((uint32_t)a.tops, a.Hkv, a.B);
  switch (a.G) {
    case 1: hipLaunchKernelGGL((block_score_kernel<1>), grid, dim3(256), 0, st, a); break;
    case 2: hipLaunchKernelGGL((block_score_kernel<2>), grid, dim3(256), 0, st, a); break;
    case 4: hipLaunchKernelGGL((block_score_kernel<4>), grid, dim3(256), 0, st, a); break;
    case 8: hipLaunchKernelGGL((block_score_kernel<8>), grid, dim3(256), 0, st, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t launch_block_select(const SelectArgs& a, hipStream_t st) {
  const dim3 grid(a.Hkv, a.B), threads(1024);
  if (a.max_blocks <= 1024) hipLaunchKernelGGL((block_select_kernel<1>), grid, threads, 0, st, a);
  else if (a.max_blocks <= 2048) hipLaunchKernelGGL((block_select_kernel<2>), grid, threads, 0, st, a);
  else if (a.max_blocks <= 4096) hipLaunchKernelGGL((block_select_kernel<4>), grid, threads, 0, st, a);
  else if (a.max_blocks <= 8192) hipLaunchKernelGGL((block_select_kernel<8>), grid, threads, 0, st, a);
  else if (a.max_blocks <= kSelectHeld) hipLaunchKernelGGL((block_select_kernel<16>), grid, threads, 0, st, a);
  else hipLaunchKernelGGL((block_select_kernel<0>), grid, threads, 0, st, a);
  return hipGetLastError();
}

}  // namespace tactic
