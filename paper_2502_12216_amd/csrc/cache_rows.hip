// Accumulated attention weights of a prompt, and what a cache keeps by them:
// eviction into another cache and the insertion of single tokens into full ones.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "common.hpp"
#include "kernels.hpp"
#include "scores.hpp"

namespace tactic {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// ---------------------------------------------------------------------------
// weights[g][j] += sum over the last `window` queries and the group's heads of
// 2^(s_ij - lse_i).  A workgroup holds 256 keys of a (sequence, KV head), 64 per
// wave, as the B operands of S = Q K^T and streams the query rows through LDS, 64
// at a time: a lane's accumulators are the rows of one key, so the sum over rows
// needs no exchange but one between the halves at the end.  Bound by the vector
// unit (one exponential, one multiply-add and one add per score, six of its slots
// where the products take four; the cap adds five); with few queries by reading K.
// Four waves that run free, two workgroups to a compute unit: eight that take turns at
// the products, as the attention's do, are slower where the vector unit has more to do
// (8192 queries, 32 heads on 8, capped: 590 us against 500; not capped 393 against 391; both before rows of NaN and left-out ones were looked for, 3%).
// grid (key tiles + sequences, Hkv, splits of the rows)
// ---------------------------------------------------------------------------
constexpr int kWKeys = 256, kWRows = 64;

template <bool kDocs>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void prompt_weights_kernel(WeightArgs a) {
  __shared__ __align__(16) unsigned char s_q[2][kWRows * 256];
  // per row: the logarithm of its sum, its slope, its position from the first key, the
  // end of the keys it sees, its document
  __shared__ __align__(16) float s_lse[2][kWRows], s_slope[2][kWRows], s_pos[2][kWRows];
  __shared__ __align__(16) int s_lim[2][kWRows], s_doc[2][kDocs ? kWRows : 4];
  __shared__ uint64_t s_odd[2];  // rows whose logarithm is NaN, or -inf (no weight)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, col = lane & 31;
  const int tid = threadIdx.x, g = blockIdx.y, split = blockIdx.z;
  int lo = 0, hi = a.B - 1;  // key tiles of sequence b start at floor(rows before it / 256) + b
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.kv_indptr[mid] / kWKeys + mid <= (int64_t)blockIdx.x) lo = mid;
    else hi = mid - 1;
  }
  const int b = lo;
  const int64_t kvb = a.kv_indptr[b];
  const int n = (int)seq_tokens(a.kv_indptr, a.seq_len, b);
  const int64_t k0l = ((int64_t)blockIdx.x - kvb / kWKeys - b) * kWKeys;
  if (k0l < 0 || k0l >= n) return;
  const int k0 = (int)k0l;
  const int64_t q0 = a.q_indptr[b];
  const int m = (int)(a.q_indptr[b + 1] - q0);
  const int pre = a.prefix_len ? a.prefix_len[b] : 0;
  // tokens [i0, m) of the sequence's queries: within the window, and able to see the tile
  int i0 = a.window > 0 ? (int)max((int64_t)m - a.window, (int64_t)0) : 0;
  if (pre <= k0) i0 = max(i0, k0 - (n - m));
  i0 = max(i0, m - n);  // queries ahead of the first token see nothing
  const int lg = a.G == 1 ? 0 : (a.G == 2 ? 1 : (a.G == 4 ? 2 : 3));
  const int rows = i0 < m ? (m - i0) << lg : 0;
  const int tiles = (rows + kWRows - 1) / kWRows;
  const int t_lo = (int)((int64_t)tiles * split / a.splits), t_hi = (int)((int64_t)tiles * (split + 1) / a.splits);

  // keys of this wave: blocks of 32, a key per column (rows past the end repeat the last)
  bf16x8 kf[2][8];
  int kdoc[2] = {0, 0};
  const int key0 = wave * 64 + col;  // from k0; the second block's: 32 more
#pragma unroll
  for (int bb = 0; bb < 2; ++bb) {
    const int key = min(k0 + key0 + bb * 32, n - 1);
    const uint16_t* at = a.K + ((int64_t)g * a.total + kvb + key) * kHeadDim + 8 * half;
    if (kDocs) kdoc[bb] = a.documents[kvb + key];
#pragma unroll
    for (int s = 0; s < 8; ++s) kf[bb][s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(at + 16 * s));
  }
  const bool capped = a.cap > 0.f, biased = a.slopes != nullptr;
  const float scale = capped ? 1.f : kInvSqrtDim * kLog2e, to_cap = capped ? kInvSqrtDim / a.cap : 0.f;
  const float cap2 = a.cap * kLog2e;
  const float keyf = (float)key0;
  float sum[2] = {0.f, 0.f};

  // documents of the key tile (from doc_range_kernel)
  const int2* dr = kDocs ? a.doc_range + (int64_t)b * a.range_stride : nullptr;
  int d_lo = 0, d_hi = 0;
  if constexpr (kDocs) {
    d_lo = INT32_MAX;
    d_hi = INT32_MIN;
    for (int t = k0 / 64; t <= min(k0 + kWKeys, n) / 64 && t * 64 < n; ++t) {
      d_lo = min(d_lo, dr[t].x);
      d_hi = max(d_hi, dr[t].y);
    }
  }
  auto next_tile = [&](int t) __attribute__((always_inline)) -> int {
    if constexpr (!kDocs) return t;
    while (t < t_hi) {
      const int mine = t + lane;
      bool some = false;
      if (mine < t_hi) {
        const int p0 = n - m + i0 + ((mine * kWRows) >> lg), p1 = n - m + i0 + ((min((mine + 1) * kWRows, rows) - 1) >> lg);
        for (int x = p0 / 64; x <= p1 / 64; ++x) some |= dr[x].x <= d_hi && dr[x].y >= d_lo;
      }
      const uint64_t any = __ballot(some);
      if (any) return t + __ffsll((unsigned long long)any) - 1;
      t += 64;
    }
    return t;
  };

  u32x4 qreg[4];
  float lse_r = 0.f, slope_r = 0.f, pos_r = 0.f;
  int lim_r = 0, doc_r = 0;
  const uint16_t* qb = a.q + ((q0 + i0) * a.Hq + (int64_t)g * a.G) * kHeadDim;
  auto fetch = [&](int t) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = (wave * 4 + i) * 64 + lane, r = c >> 4, row = min(t * kWRows + r, rows - 1);
      const int64_t at = ((int64_t)(row >> lg) * a.Hq + (row & (a.G - 1))) * kHeadDim;
      qreg[i] = *reinterpret_cast<const u32x4*>(qb + at + ((c & 15) ^ (4 * (r & 3) + ((r >> 2) & 3))) * 8);
    }
    if (tid < kWRows) {
      const int x = t * kWRows + tid, row = min(x, rows - 1), i = i0 + (row >> lg), h = g * a.G + (row & (a.G - 1));
      const int pos = n - m + i;
      const float l = a.lse[(int64_t)h * a.n_queries + q0 + i];
      // a row past the end, and one whose sum says that it saw nothing, gives no weight and
      // sees no key, whatever the row holds
      lse_r = x < rows ? l * kLog2e : INFINITY;  // (NaN and -inf stay)
      slope_r = biased ? a.slopes[h] * kLog2e / scale : 0.f;
      pos_r = (float)(pos - k0);
      lim_r = x >= rows || l == -INFINITY ? INT32_MIN : min(max(pos + 1, pre), n) - k0;
      if (kDocs) doc_r = a.documents[kvb + max(pos, 0)];
    }
  };
  auto store = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<u32x4*>(s_q[buf] + ((wave * 4 + i) * 64 + lane) * 16) = qreg[i];
    if (tid < kWRows) {
      const uint64_t odd_rows = __ballot(!(lse_r > -INFINITY));
      if (tid == 0) s_odd[buf] = odd_rows;
      s_lse[buf][tid] = lse_r > -INFINITY ? lse_r : (lse_r == -INFINITY ? INFINITY : 0.f);
      s_slope[buf][tid] = slope_r;
      s_pos[buf][tid] = pos_r;
      s_lim[buf][tid] = lim_r;
      if (kDocs) s_doc[buf][tid] = doc_r;
    }
  };
  const uint32_t q_off = col * 256 + ((half ^ (4 * (col & 3) + ((col >> 2) & 3))) * 16);
  int t = next_tile(t_lo);
  if (t < t_hi) {
    fetch(t);
    store(0);
  }
  __syncthreads();
  int buf = 0;
  while (t < t_hi) {
    const int tn = next_tile(t + 1);
    if (tn < t_hi) fetch(tn);
    const bool odd = __builtin_amdgcn_readfirstlane((int)(s_odd[buf] != 0));
    if (odd) {
      // rare: a row of NaN gives NaN to the keys it sees, by its scores, which the masks leave out
      if (tid < kWRows && (s_odd[buf] >> tid & 1) && s_lse[buf][tid] != INFINITY)
        *reinterpret_cast<uint32_t*>(s_q[buf] + tid * 256) = 0x7fff7fffu;
      __syncthreads();
    }
    // the first token of the tile sees the fewest keys
    const int lim0 = min(max(n - m + i0 + ((t * kWRows) >> lg) + 1, pre), n);
    const bool masked = kDocs || odd || k0 + wave * 64 + 64 > lim0;
#pragma unroll
    for (int rb = 0; rb < 2; ++rb) {
      f32x16 acc[2];
#pragma unroll
      for (int bb = 0; bb < 2; ++bb)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[bb][r] = 0.f;
      uint32_t off = q_off + buf * (kWRows * 256) + rb * 8192;
      asm volatile("" : "+v"(off));
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        const bf16x8 qv = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(s_q[0] + (off ^ (s * 32))));
        acc[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qv, kf[0][s], acc[0], 0, 0, 0);
        acc[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qv, kf[1][s], acc[1], 0, 0, 0);
      }
      // accumulator r is row rb * 32 + 8 (r / 4) + 4 half + r % 4
      const int at = rb * 32 + 4 * half;
      if (capped) {
        float big = 0.f;
#pragma unroll
        for (int bb = 0; bb < 2; ++bb)
#pragma unroll
          for (int r = 0; r < 16; ++r) big = fmaxf(big, fabsf(acc[bb][r]));
        if (!__any(big > a.poly.near)) {
#pragma unroll
          for (int bb = 0; bb < 2; ++bb)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              acc[bb][r] = cap_near(acc[bb][r], a.poly);
              if (r % 8 == 7) __builtin_amdgcn_sched_barrier(0);
            }
        } else if (!__any(big > a.poly.far)) {
#pragma unroll
          for (int bb = 0; bb < 2; ++bb)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              acc[bb][r] = cap_far(acc[bb][r], a.poly);
              if (r % 8 == 7) __builtin_amdgcn_sched_barrier(0);
            }
        } else {
#pragma unroll
          for (int bb = 0; bb < 2; ++bb)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              acc[bb][r] = cap2 * tanh_any(acc[bb][r] * to_cap);
              if (r % 2) __builtin_amdgcn_sched_barrier(0);
            }
        }
      }
      if (biased) {
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          const float4 sl = *reinterpret_cast<const float4*>(s_slope[buf] + at + 2 * r);
          const float4 ps = *reinterpret_cast<const float4*>(s_pos[buf] + at + 2 * r);
          const float sla[4] = {sl.x, sl.y, sl.z, sl.w}, psa[4] = {ps.x, ps.y, ps.z, ps.w};
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int bb = 0; bb < 2; ++bb) acc[bb][r + j] = fmaf(-sla[j], fabsf(psa[j] - keyf - 32.f * bb), acc[bb][r + j]);
        }
      }
      if (masked) {
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          const int4 lm = *reinterpret_cast<const int4*>(s_lim[buf] + at + 2 * r);
          const int lma[4] = {lm.x, lm.y, lm.z, lm.w};
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int bb = 0; bb < 2; ++bb) acc[bb][r + j] = key0 + 32 * bb < lma[j] ? acc[bb][r + j] : -INFINITY;
          if constexpr (kDocs) {
            const int4 dc = *reinterpret_cast<const int4*>(s_doc[buf] + at + 2 * r);
            const int dca[4] = {dc.x, dc.y, dc.z, dc.w};
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
              for (int bb = 0; bb < 2; ++bb) acc[bb][r + j] = dca[j] == kdoc[bb] ? acc[bb][r + j] : -INFINITY;
          }
        }
      }
      float part[2][2] = {{0.f, 0.f}, {0.f, 0.f}};
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const float4 ls = *reinterpret_cast<const float4*>(s_lse[buf] + at + 2 * r);
        const float lsa[4] = {ls.x, ls.y, ls.z, ls.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int bb = 0; bb < 2; ++bb) part[bb][j & 1] += fast_exp2(fmaf(acc[bb][r + j], scale, -lsa[j]));
      }
#pragma unroll
      for (int bb = 0; bb < 2; ++bb) sum[bb] += part[bb][0] + part[bb][1];
    }
    if (tn < t_hi) store(buf ^ 1);
    __syncthreads();
    buf ^= 1;
    t = tn;
  }
#pragma unroll
  for (int bb = 0; bb < 2; ++bb) {
    const float s = sum[bb] + __shfl_xor(sum[bb], 32, 64);
    const int key = k0 + key0 + bb * 32;
    if (half == 0 && key < n) {
      const int64_t at = (int64_t)g * a.total + kvb + key;
      if (a.splits == 1) a.weights[at] += s;
      else a.part[(int64_t)split * a.Hkv * a.total + at] = s;
    }
  }
}

// Adds the splits' sums in order.  grid (rows / 256, Hkv, B)
__global__ __launch_bounds__(256) void sum_weights_kernel(WeightArgs a) {
  const int g = blockIdx.y, b = blockIdx.z;
  const int64_t n = seq_tokens(a.kv_indptr, a.seq_len, b), r = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (r >= n) return;
  const int64_t at = (int64_t)g * a.total + a.kv_indptr[b] + r;
  float x = 0.f;
  for (int s = 0; s < a.splits; ++s) x += a.part[(int64_t)s * a.Hkv * a.total + at];
  a.weights[at] += x;
}

hipError_t launch_prompt_weights(const WeightArgs& a, int64_t max_len, hipStream_t st) {
  if (max_len == 0) return hipSuccess;
  const dim3 grid((unsigned)(a.total / kWKeys + a.B), a.Hkv, a.splits);
  if (a.documents) hipLaunchKernelGGL(prompt_weights_kernel<true>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(prompt_weights_kernel<false>, grid, dim3(256), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && a.splits > 1) {
    hipLaunchKernelGGL(sum_weights_kernel, dim3((unsigned)((max_len + 255) / 256), a.Hkv, a.B), dim3(256), 0, st, a);
    e = hipGetLastError();
  }
  return e;
}

// ---------------------------------------------------------------------------
// Which rows stay.  Rows are ranked by a 32-bit key: weights ascending (-0 as 0,
// NaN below every number), above them the recent rows by position.  Among equal
// keys the lower row ranks first.
// ---------------------------------------------------------------------------
constexpr uint32_t kRecentKey = 0xff800001u;  // above the key of +inf

__device__ __forceinline__ uint32_t rank_key(float w, int pos, int newest, int recent) {
  const uint32_t age = pos >= newest ? 0u : (uint32_t)newest - (uint32_t)pos;  // 0: the newest
  const uint32_t u = __float_as_uint(w + 0.f), flip = (uint32_t)((int)u >> 31) | 0x80000000u;
  const uint32_t by_weight = w != w ? 0u : u ^ flip;
  return age < (uint32_t)recent ? kRecentKey + (uint32_t)(recent - 1) - age : by_weight;
}

struct __attribute__((packed, aligned(4))) Four {  // 16 bytes at any 4-byte place
  uint32_t v[4];
};

// Keys of rows r .. r + 3.  Past the end 0, the least: fewer than n rows are kept and the
// lower row goes first, so that no such row ever is.
__device__ __forceinline__ void rank_keys(const float* w, const int32_t* pos, int n, int newest, int recent, int64_t r,
                                          uint32_t (&k)[4]) {
  if (r + 4 <= n) {
    const Four x = *reinterpret_cast<const Four*>(w + r);
    Four p = {{0, 0, 0, 0}};
    if (pos) p = *reinterpret_cast<const Four*>(pos + r);
#pragma unroll
    for (int e = 0; e < 4; ++e) k[e] = rank_key(__uint_as_float(x.v[e]), pos ? (int)p.v[e] : (int)r + e, newest, recent);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) k[e] = r + e < n ? rank_key(w[r + e], pos ? pos[r + e] : (int)r + e, newest, recent) : 0u;
  }
}
// Adds one to the count of `bin` in LDS.  Lanes of one bin take turns, so that those of
// the first lane's bin are counted at once (one workgroup on 65536 + 30011 equal rows, 8 KV
// heads: 80 us a call so, half of it the copy, 229 with one atomic per row; power law 72, 78).
__device__ __forceinline__ void count_key(uint32_t* hist, bool in, uint32_t bin, int lane) {
  const uint64_t left = __ballot(in);
  if (left == 0) return;
  const int lead = __ffsll((unsigned long long)left) - 1;
  const uint32_t of = (uint32_t)__builtin_amdgcn_readlane((int)bin, lead);
  const uint64_t same = __ballot(in && bin == of);
  const uint32_t add = lane == lead ? (uint32_t)__popcll(same) : 1u;
  if (in && (lane == lead || bin != of)) atomicAdd(&hist[bin], add);
}
// Sum of one value per thread over the threads before it (1024 of them), and of all.
__device__ __forceinline__ uint32_t scan_1024(uint32_t* s_sum, uint32_t x, int lane, int wave, uint32_t* all) {
  const uint32_t incl = (uint32_t)wave_incl_scan((int)x);
  if (lane == kWave - 1) s_sum[wave] = incl;
  __syncthreads();
  uint32_t before = 0, total = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint32_t v = s_sum[i];
    before += i < wave ? v : 0;
    total += v;
  }
  __syncthreads();
  if (all) *all = total;
  return before + incl - x;
}

// One workgroup per (KV head, sequence) finds the kept rows: the key of the last kept
// one digit by digit (11, 11 and 10 bits), then the kept rows in ascending order.
// Thread t holds rows 4 (1024 j + t) + e, e < 4, j < J, as keys in registers, so that
// weights and positions are read once (J = 16: 65536 rows, 38 us); J = 0 makes the keys again
// in every pass (131072 rows: about 110 us).  Bound by one compute unit's reads and counts: the digits' counts are
// LDS atomics, of which those on one count take turns.
template <int J>
__global__ __launch_bounds__(1024) void evict_select_kernel(EvictArgs a) {
  constexpr int kBins = 2048, kHeld = J > 0 ? J : 1;
  __shared__ uint32_t s_hist[kBins];
  __shared__ uint32_t s_sum[16];
  __shared__ uint32_t s_prefix, s_need, s_same;
  const int g = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t kvb = a.kv_indptr[b], outb = a.out_indptr[b];
  const int n = (int)seq_tokens(a.kv_indptr, a.seq_len, b);
  const int64_t room = a.out_indptr[b + 1] - outb;
  const int keep = (int)min((int64_t)n, min(max((int64_t)a.keep[b], (int64_t)0), room));
  if (g == 0 && tid == 0) a.out_len[b] = keep;
  if (keep == 0) return;
  const int newest = a.newest ? a.newest[b] : n - 1;
  const float* w = a.weights + (int64_t)g * a.total + kvb;
  const int32_t* pos = a.positions ? a.positions + (int64_t)g * a.total + kvb : nullptr;
  int32_t* rows = a.rows + (int64_t)g * a.out_total + outb;
  if (keep == n) {
    for (int r = tid; r < n; r += 1024) rows[r] = r;
    return;
  }
  auto keys_at = [&](int64_t r, uint32_t (&k)[4]) __attribute__((always_inline)) {
    rank_keys(w, pos, n, newest, a.recent, r, k);
  };
  const int steps = (int)(((int64_t)n + 4095) / 4096);  // of 4096 rows
  uint32_t held[kHeld][4];
  if constexpr (J > 0) {
#pragma unroll
    for (int j = 0; j < J; ++j) keys_at((int64_t)j * 4096 + tid * 4, held[j]);
  }
  auto count = [&](bool in, uint32_t bin) __attribute__((always_inline)) { count_key(s_hist, in, bin, lane); };
  // f(row, its four keys) for every step of the thread's rows
  auto each = [&](auto f) __attribute__((always_inline)) {
    if constexpr (J > 0) {
#pragma unroll
      for (int j = 0; j < J; ++j)
        if (j < steps) f((int64_t)j * 4096 + tid * 4, held[j]);
    } else {
      for (int j = 0; j < steps; ++j) {
        uint32_t k[4];
        keys_at((int64_t)j * 4096 + tid * 4, k);
        f((int64_t)j * 4096 + tid * 4, k);
      }
    }
  };
  auto scan = [&](uint32_t x, uint32_t* all) __attribute__((always_inline)) { return scan_1024(s_sum, x, lane, wave, all); };
  uint32_t prefix = 0, need = (uint32_t)keep;
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0), bits = pass == 2 ? 10 : 11;
    s_hist[tid] = 0;
    s_hist[tid + 1024] = 0;
    __syncthreads();
    each([&](int64_t r, const uint32_t (&k)[4]) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        count(pass == 0 || (k[e] >> (shift + bits)) == (prefix >> (shift + bits)), (k[e] >> shift) & ((1u << bits) - 1));
    });
    __syncthreads();
    // the digit that holds the need-th largest: two counts per thread from the top
    const uint32_t c0 = s_hist[kBins - 1 - 2 * tid], c1 = s_hist[kBins - 2 - 2 * tid];
    const uint32_t before = scan(c0 + c1, nullptr);
    if (before < need && need <= before + c0 + c1) {
      const bool second = need > before + c0;
      s_prefix = prefix | ((uint32_t)(kBins - 1 - 2 * tid - (second ? 1 : 0)) << shift);
      s_need = need - before - (second ? c0 : 0);
      s_same = second ? c1 : c0;
    }
    __syncthreads();
    prefix = s_prefix;
    need = s_need;
  }
  // rows above the key stay, and the first `need` of the s_same rows of exactly that key
  const bool ties = s_same != need;
  __syncthreads();
  if constexpr (J > 0) {
    // counts of every step first: one scan over (step, wave) gives every thread's places
    auto places = [&](const uint32_t (&cnt)[kHeld], uint32_t (&at)[kHeld]) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const uint32_t incl = (uint32_t)wave_incl_scan((int)cnt[j]);
        if (lane == kWave - 1) s_hist[j * 16 + wave] = incl;
        at[j] = incl - cnt[j];
      }
      __syncthreads();
      const uint32_t x = tid < J * 16 ? s_hist[tid] : 0, before = scan(x, nullptr);
      if (tid < J * 16) s_hist[tid] = before;
      __syncthreads();
#pragma unroll
      for (int j = 0; j < J; ++j) at[j] += s_hist[j * 16 + wave];
      __syncthreads();
    };
    uint32_t kept[kHeld], cnt[kHeld], at[kHeld];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      uint32_t above = 0, eq = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        above |= (uint32_t)(held[j][e] > prefix) << e;
        eq |= (uint32_t)(held[j][e] == prefix) << e;
      }
      kept[j] = above | (ties ? eq << 4 : eq);  // (bits 4 to 7: equal ones, not decided yet)
      cnt[j] = __popc(eq);
    }
    if (ties) {
      places(cnt, at);
#pragma unroll
      for (int j = 0; j < J; ++j) {
        uint32_t rank = at[j], take = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t is = kept[j] >> (4 + e) & 1;
          take |= (is && rank < need ? 1u : 0u) << e;
          rank += is;
        }
        kept[j] = (kept[j] & 15u) | take;
      }
    }
#pragma unroll
    for (int j = 0; j < J; ++j) cnt[j] = __popc(kept[j]);
    places(cnt, at);
#pragma unroll
    for (int j = 0; j < J; ++j) {
      uint32_t to = at[j];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (kept[j] >> e & 1) {
          if (to < (uint32_t)keep) rows[to] = j * 4096 + tid * 4 + e;
          ++to;
        }
    }
    return;
  }
  uint32_t base = 0, eq_base = 0;
  each([&](int64_t r, const uint32_t (&k)[4]) {
    uint32_t kept = 0, eq = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      kept |= (uint32_t)(k[e] > prefix) << e;
      eq |= (uint32_t)(k[e] == prefix) << e;
    }
    if (ties) {
      uint32_t all;
      uint32_t rank = eq_base + scan(__popc(eq), &all);
      eq_base += all;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        kept |= (uint32_t)((eq >> e & 1) && rank < need) << e;
        rank += eq >> e & 1;
      }
    } else {
      kept |= eq;
    }
    uint32_t all;
    uint32_t at = base + scan(__popc(kept), &all);
    base += all;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (kept >> e & 1) {
        if (at < (uint32_t)keep) rows[at] = (int32_t)(r + e);
        ++at;
      }
  });
}

// The same by several workgroups for a (KV head, sequence), each with a slice of the rows,
// in four launches: launch P < 3 counts digit P of the slice's keys that have the digits
// found so far, launch P > 0 first adds the slices' counts of digit P - 1 and finds it, all
// of them alike, and what of it lies in the slices before.  The last one places the rows.
// Bound by the launches' chains, each 5 to 8 us (16 slices' counts are 128 KB to read).
// grid (slices, Hkv, B)
template <int P>
__global__ __launch_bounds__(1024) void evict_slice_kernel(EvictArgs a) {
  __shared__ uint32_t s_hist[kEvictBins];
  __shared__ uint32_t s_sum[16], s_ahead[16];
  __shared__ uint32_t s_prefix, s_need, s_same, s_before;
  const int slice = blockIdx.x, g = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t kvb = a.kv_indptr[b], outb = a.out_indptr[b];
  const int n = (int)seq_tokens(a.kv_indptr, a.seq_len, b);
  const int64_t room = a.out_indptr[b + 1] - outb;
  const int keep = (int)min((int64_t)n, min(max((int64_t)a.keep[b], (int64_t)0), room));
  if (P == 3 && slice == 0 && g == 0 && tid == 0) a.out_len[b] = keep;
  const int steps = (int)(((int64_t)n + 4096 * kEvictSlices - 1) / (4096 * kEvictSlices));  // of 4096 rows
  const int64_t r0 = (int64_t)slice * steps * 4096, r1 = min(r0 + (int64_t)steps * 4096, (int64_t)n);
  if (keep == 0 || r0 >= n) return;
  int32_t* rows = a.rows + (int64_t)g * a.out_total + outb;
  if (keep == n) {
    if (P == 3)
      for (int64_t r = r0 + tid; r < r1; r += 1024) rows[r] = (int32_t)r;
    return;
  }
  const int newest = a.newest ? a.newest[b] : n - 1;
  const float* w = a.weights + (int64_t)g * a.total + kvb;
  const int32_t* pos = a.positions ? a.positions + (int64_t)g * a.total + kvb : nullptr;
  const int64_t groups = (int64_t)a.B * a.Hkv, group = (int64_t)b * a.Hkv + g;
  auto counts_of = [&](int pass, int s) __attribute__((always_inline)) {
    return a.counts + (((int64_t)pass * groups + group) * kEvictSlices + s) * kEvictBins;
  };
  uint32_t prefix = 0, need = (uint32_t)keep, ahead = 0, eq_ahead = 0;
  bool ties = false;
  if constexpr (P > 0) {
    constexpr int shift = P == 1 ? 21 : (P == 2 ? 10 : 0);
    if constexpr (P > 1) {
      const uint2 c = a.chosen[(P - 2) * groups + group];
      prefix = c.x;
      need = c.y;
      ahead = a.ahead[((P - 2) * groups + group) * kEvictSlices + slice];
    }
    const int used = (int)(((int64_t)n + (int64_t)steps * 4096 - 1) / ((int64_t)steps * 4096));
    // two counts per thread from the top: of all slices, and of those before this one
    uint32_t c0 = 0, c1 = 0, m0 = 0, m1 = 0;
    uint2 c[kEvictSlices];
#pragma unroll
    for (int s = 0; s < kEvictSlices; ++s)
      c[s] = s < used ? *reinterpret_cast<const uint2*>(counts_of(P - 1, s) + kEvictBins - 2 - 2 * tid) : make_uint2(0, 0);
#pragma unroll
    for (int s = 0; s < kEvictSlices; ++s) {
      c0 += c[s].y;
      c1 += c[s].x;
      m0 += s < slice ? c[s].y : 0;
      m1 += s < slice ? c[s].x : 0;
    }
    const uint32_t before = scan_1024(s_sum, c0 + c1, lane, wave, nullptr);
    const bool mine = before < need && need <= before + c0 + c1, second = need > before + c0;
    if (mine) {
      s_prefix = prefix | ((uint32_t)(kEvictBins - 1 - 2 * tid - (second ? 1 : 0)) << shift);
      s_need = need - before - (second ? c0 : 0);
      s_same = second ? c1 : c0;
      s_before = second ? m1 : m0;
    }
    // rows of larger digits in the slices before: whole threads before the digit's, and its first count
    uint32_t larger = before + c0 + c1 < need ? m0 + m1 : (mine && second ? m0 : 0);
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) larger += __shfl_xor(larger, s, 64);
    if (lane == 0) s_ahead[wave] = larger;
    __syncthreads();
    prefix = s_prefix;
    need = s_need;
    ties = s_same != need;
    eq_ahead = s_before;
#pragma unroll
    for (int i = 0; i < 16; ++i) ahead += s_ahead[i];
    if (P < 3 && tid == 0) {
      a.ahead[((P - 1) * groups + group) * kEvictSlices + slice] = ahead;
      if (slice == 0) a.chosen[(P - 1) * groups + group] = make_uint2(prefix, need);
    }
  }
  if constexpr (P < 3) {
    constexpr int shift = P == 0 ? 21 : (P == 1 ? 10 : 0), bits = P == 2 ? 10 : 11;
    s_hist[tid] = 0;
    s_hist[tid + 1024] = 0;
    __syncthreads();
    for (int64_t r = r0 + tid * 4; r < r0 + (int64_t)steps * 4096; r += 4096) {
      uint32_t k[4];
      rank_keys(w, pos, n, newest, a.recent, r, k);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        count_key(s_hist, P == 0 || (k[e] >> (shift + bits)) == (prefix >> (shift + bits)), (k[e] >> shift) & ((1u << bits) - 1), lane);
    }
    __syncthreads();
    *reinterpret_cast<uint2*>(counts_of(P, slice) + 2 * tid) = make_uint2(s_hist[2 * tid], s_hist[2 * tid + 1]);
  } else {
    // rows above the key stay, and the first `need` of those of exactly that key
    uint32_t at0 = ahead + min(eq_ahead, need), eq0 = eq_ahead;
    for (int64_t r = r0 + tid * 4; r < r0 + (int64_t)steps * 4096; r += 4096) {
      uint32_t k[4], kept = 0, eq = 0, all;
      rank_keys(w, pos, n, newest, a.recent, r, k);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        kept |= (uint32_t)(k[e] > prefix) << e;
        eq |= (uint32_t)(k[e] == prefix) << e;
      }
      if (ties) {
        uint32_t rank = eq0 + scan_1024(s_sum, __popc(eq), lane, wave, &all);
        eq0 += all;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          kept |= (uint32_t)((eq >> e & 1) && rank < need) << e;
          rank += eq >> e & 1;
        }
      } else {
        kept |= eq;
      }
      uint32_t at = at0 + scan_1024(s_sum, __popc(kept), lane, wave, &all);
      at0 += all;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (kept >> e & 1) {
          if (at < (uint32_t)keep) rows[at] = (int32_t)(r + e);
          ++at;
        }
    }
  }
}

// Copies the kept rows: 16 lanes per row, K and V.  grid (rows / 64, Hkv, B).  Bound by
// HBM, the read rows being 256 bytes each (23884 rows x 8 heads, 196 MB read and written:
// 35 us, 5.6 TB/s).
__global__ __launch_bounds__(256) void evict_gather_kernel(EvictArgs a) {
  const int g = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, part = tid & 15;
  const int64_t kvb = a.kv_indptr[b], outb = a.out_indptr[b], keep = a.out_len[b];
  const int64_t base = (int64_t)blockIdx.x * 64;
  if (base >= keep) return;
  const int32_t* rows = a.rows + (int64_t)g * a.out_total + outb;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t at = base + i * 16 + (tid >> 4);
    if (at >= keep) continue;
    const int64_t r = rows[at];
    const int64_t from = (int64_t)g * a.total + kvb + r, to = (int64_t)g * a.out_total + outb + at;
    const uint4 k = *reinterpret_cast<const uint4*>(a.K + from * kHeadDim + part * 8);
    const uint4 v = *reinterpret_cast<const uint4*>(a.V + from * kHeadDim + part * 8);
    *reinterpret_cast<uint4*>(a.K_out + to * kHeadDim + part * 8) = k;
    *reinterpret_cast<uint4*>(a.V_out + to * kHeadDim + part * 8) = v;
    if (part == 0) {
      a.weights_out[to] = a.weights[from];
      a.positions_out[to] = a.positions ? a.positions[from] : (int32_t)r;
    }
  }
}

hipError_t launch_evict(const EvictArgs& a, int64_t max_len, int64_t max_out, hipStream_t st) {
  const dim3 grid(a.Hkv, a.B), slices(kEvictSlices, a.Hkv, a.B);
  if (a.counts) {
    hipLaunchKernelGGL(evict_slice_kernel<0>, slices, dim3(1024), 0, st, a);
    hipLaunchKernelGGL(evict_slice_kernel<1>, slices, dim3(1024), 0, st, a);
    hipLaunchKernelGGL(evict_slice_kernel<2>, slices, dim3(1024), 0, st, a);
    hipLaunchKernelGGL(evict_slice_kernel<3>, slices, dim3(1024), 0, st, a);
  } else if (max_len <= 4096) hipLaunchKernelGGL(evict_select_kernel<1>, grid, dim3(1024), 0, st, a);
  else if (max_len <= 16384) hipLaunchKernelGGL(evict_select_kernel<4>, grid, dim3(1024), 0, st, a);
  else if (max_len <= 65536) hipLaunchKernelGGL(evict_select_kernel<16>, grid, dim3(1024), 0, st, a);
  else hipLaunchKernelGGL(evict_select_kernel<0>, grid, dim3(1024), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && max_out > 0) {
    hipLaunchKernelGGL(evict_gather_kernel, dim3((unsigned)((max_out + 63) / 64), a.Hkv, a.B), dim3(256), 0, st, a);
    e = hipGetLastError();
  }
  return e;
}

// ---------------------------------------------------------------------------
// One token per sequence: behind the last row while there is room, else in the
// place of the row that ranks last.  One workgroup per (KV head, sequence), a thread for
// four rows at a time; bound by its chain of loads, reduction and stores (full caches of
// 4 x 16384 rows, 8 KV heads: 7.9 us with the launch that sets the lengths, which waits
// for every head; with one row at a time and 256 threads 20).
// ---------------------------------------------------------------------------
// Lowest key of rows [0, n), with the highest row of it among equal ones, over the
// threads whose four-row pieces start at `first`, `step` rows apart: (key, ~row).
__device__ __forceinline__ uint64_t least_row(const InsertArgs& a, int64_t base, int n, int newest, int64_t first, int step) {
  uint64_t best = ~0ull;
#pragma unroll 2
  for (int64_t r = first; r < n; r += step) {
    uint32_t k[4];
    rank_keys(a.weights + base, a.positions + base, n, newest, a.recent, r, k);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (r + e < n) best = min(best, ((uint64_t)k[e] << 32) | (uint32_t)~(uint32_t)(r + e));
  }
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) best = min(best, (uint64_t)__shfl_xor((unsigned long long)best, s, 64));
  return best;
}

__global__ __launch_bounds__(1024) void insert_token_kernel(InsertArgs a) {
  __shared__ uint64_t s_min[16];
  const int g = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t kvb = a.kv_indptr[b], span = a.kv_indptr[b + 1] - kvb;
  const int n = (int)seq_tokens(a.kv_indptr, a.seq_len, b);
  const int64_t base = (int64_t)g * a.total + kvb;
  int64_t row = n;
  if (span == 0) {
    if (tid == 0) a.rows[(int64_t)b * a.Hkv + g] = -1;
    return;
  }
  if (n >= span) {
    uint64_t best = least_row(a, base, n, a.newest[b], tid * 4, 4096);
    if (lane == 0) s_min[wave] = best;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 16; ++i) best = min(best, s_min[i]);
    row = (int64_t)(uint32_t)~(uint32_t)best;
  }
  const int64_t from = ((int64_t)b * a.Hkv + g) * kHeadDim, to = (base + row) * kHeadDim;
  if (tid < 16) *reinterpret_cast<uint4*>(a.K + to + tid * 8) = *reinterpret_cast<const uint4*>(a.k + from + tid * 8);
  else if (tid < 32) *reinterpret_cast<uint4*>(a.V + to + (tid - 16) * 8) = *reinterpret_cast<const uint4*>(a.v + from + (tid - 16) * 8);
  else if (tid == 32) {
    a.weights[base + row] = 0.f;
    a.positions[base + row] = a.newest[b];
    a.rows[(int64_t)b * a.Hkv + g] = (int32_t)row;
  }
}

__global__ __launch_bounds__(256) void advance_lengths_kernel(InsertArgs a) {
  const int b = blockIdx.x * 256 + threadIdx.x;
  if (b < a.B) {
    const int64_t span = a.kv_indptr[b + 1] - a.kv_indptr[b];
    a.seq_len[b] = min(max(a.seq_len[b], (int64_t)0) + 1, span);
  }
}

// The same with one workgroup per sequence, its waves shared out among the heads, which
// sets the length itself behind a barrier (16 full sequences of 2048 rows, 8 KV heads: 6.6 to 7.1 us).
__global__ __launch_bounds__(1024) void insert_heads_kernel(InsertArgs a) {
  __shared__ uint64_t s_min[16];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int waves = 16 / a.Hkv, g = wave / waves, part = wave % waves;  // (Hkv <= 16)
  const int64_t kvb = a.kv_indptr[b], span = a.kv_indptr[b + 1] - kvb;
  const int n = (int)seq_tokens(a.kv_indptr, a.seq_len, b), newest = a.newest[b];
  const int64_t base = (int64_t)g * a.total + kvb;
  uint64_t best = ~0ull;
  if (n >= span && g < a.Hkv) best = least_row(a, base, n, newest, (part * 64 + lane) * 4, waves * 256);
  if (lane == 0) s_min[wave] = best;
  __syncthreads();  // (and every wave has read the length)
  if (tid == 0) a.seq_len[b] = min((int64_t)n + 1, span);
  if (g >= a.Hkv || part != 0) return;
  for (int i = 1; i < waves; ++i) best = min(best, s_min[wave + i]);
  const int64_t row = n < span ? n : (int64_t)(uint32_t)~(uint32_t)best;
  const int64_t from = ((int64_t)b * a.Hkv + g) * kHeadDim, to = (base + row) * kHeadDim;
  if (lane == 32) a.rows[(int64_t)b * a.Hkv + g] = span == 0 ? -1 : (int32_t)row;
  if (span == 0) return;
  if (lane < 16) *reinterpret_cast<uint4*>(a.K + to + lane * 8) = *reinterpret_cast<const uint4*>(a.k + from + lane * 8);
  else if (lane < 32) *reinterpret_cast<uint4*>(a.V + to + (lane - 16) * 8) = *reinterpret_cast<const uint4*>(a.v + from + (lane - 16) * 8);
  else if (lane == 32) {
    a.weights[base + row] = 0.f;
    a.positions[base + row] = newest;
  }
}

hipError_t launch_insert(const InsertArgs& a, int64_t max_len, hipStream_t st) {
  // One launch or two, us a call in a stream and in a graph: 2 heads of 1000 rows 10.0, 3.6 and
  // 12.2, 5.1; 8 of 2048 10.3, 6.6 and 12.5, 5.5; 8 of 4096 10.3, 8.9 and 12.4, 5.7; 8 of 8192 14.5,
  // 14.4 and 12.1, 6.5.  In a stream the second launch costs the host 2 us up to 8 of 4096, in
  // a graph the one launch's compute unit is the slower from 8 of about 1500 on: the limit lies
  // between, where the one gains 2.2 in a stream and loses 1.1 in a graph.
  if (a.Hkv <= 16 && max_len * a.Hkv <= 16384) {
    hipLaunchKernelGGL(insert_heads_kernel, dim3(a.B), dim3(1024), 0, st, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(insert_token_kernel, dim3(a.Hkv, a.B), dim3(1024), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess) {
    hipLaunchKernelGGL(advance_lengths_kernel, dim3((a.B + 255) / 256), dim3(256), 0, st, a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace tactic
