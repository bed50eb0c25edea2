// Rows into a cache of 8 or 4 bits, with the bounds of their blocks, and out of it.
//
// Both move bytes: a row of K or V is 256 bytes in bf16 and 132 or 68 in the cache.  16
// lanes share a row, 8 values each, so that a group of 32 is four lanes and its largest
// value two DPP steps; nothing is read twice but the rows of a block that was begun
// before, whose bounds are taken again from the cache.  8 KV heads: 33193 rows to 4 bits with
// bounds, in pages, 40 us (4.4 TB/s; without bounds 33 to 35: the vector unit shows), 131072
// rows to 8 bits with bounds 136 (6.0 TB/s); 65536 rows of 8 bits back to bf16 68 us (5.9 TB/s);
// a token for each of 32 sequences 5.6 us, a chain of four loads.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.hpp"
#include "kernels.hpp"
#include "quant.hpp"

namespace tactic {

// A work item's sequence and what is known of it, the same in all lanes.
struct Source {
  int b;
  int64_t first, rows, kvb, n;  // its rows among all, how many; its span's start, its length
};

// The sequence of work item `item` where the items of one that starts at row r of all are from
// r / kRows + extra b on: 64 sequences looked at in one step, a lane each, with all that
// is read of them loaded at once.
template <int kRows, int kExtra>
__device__ __forceinline__ Source source_of(const QuantRowsArgs& a, int64_t item) {
  const int lane = threadIdx.x & (kWave - 1);
  Source s{};
  for (int b0 = 0; b0 < a.B; b0 += kWave) {
    const int b = min(b0 + lane, a.B - 1);
    const int64_t r0 = a.row_indptr[b], r1 = a.row_indptr[b + 1], k0 = a.kv_indptr[b], k1 = a.kv_indptr[b + 1];
    const int64_t len = a.seq_len ? a.seq_len[b] : k1 - k0;
    const int n = __popcll(__ballot(b0 + lane < a.B && r0 / kRows + kExtra * (int64_t)b <= item));
    if (n > 0) {
      auto of = [&](int64_t x) {
        return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), n - 1) << 32 |
                         (uint32_t)__builtin_amdgcn_readlane((int)x, n - 1));
      };
      s.b = b0 + n - 1;
      s.first = of(r0);
      s.rows = of(r1 - r0);
      s.kvb = of(k0);
      s.n = of(max((int64_t)0, min(len, k1 - k0)));
    }
    if (n < kWave) break;
  }
  s.b = __builtin_amdgcn_readfirstlane(s.b);
  return s;
}

// Index of sequence row `row` among the rows of [Hkv][total] or [num_pages][Hkv][page_size];
// -1: a page that is not there
__device__ __forceinline__ int64_t place_of(const QuantKV& kv, int Hkv, int64_t total, int64_t kvb, int b, int g, int row) {
  if (!kv.paged) return (int64_t)g * total + kvb + row;
  const int size = kv.pk.page_size;
  // (sizes are powers of two as a rule: a division is 20 instructions)
  const int at = (size & (size - 1)) == 0 ? row >> __builtin_ctz(size) : row / size;
  const int page = kv.pk.page_table[(int64_t)b * kv.pk.max_pages + min(at, kv.pk.max_pages - 1)];
  if (page < 0 || page >= kv.pk.num_pages) return -1;
  return (int64_t)((page * Hkv + g) * size + (row - at * size));  // (fewer than 2^31 rows)
}

template <int kBits>
__device__ __forceinline__ uint2 load_codes(const uint8_t* p) {
  if constexpr (kBits == 8) return *reinterpret_cast<const uint2*>(p);
  else return make_uint2(*reinterpret_cast<const uint32_t*>(p), 0u);
}

__device__ __forceinline__ uint32_t pk_max(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
// Largest |bf16| of a group, as its bits, from the words of four lanes
__device__ __forceinline__ uint32_t largest(const uint4& x) {
  uint32_t t = pk_max(pk_max(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), pk_max(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu));
  t = pk_max(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0x4E, 0xF, 0xF, false));
  t = pk_max(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0xB1, 0xF, 0xF, false));
  return max(t & 0xffffu, t >> 16);
}
// Two bf16 as 16-bit integers that order as they do, and back: an involution
__device__ __forceinline__ uint32_t ordered(uint32_t w) {
  const i16x2 x = __builtin_bit_cast(i16x2, w);
  return w ^ (__builtin_bit_cast(uint32_t, x >> 15) & 0x7fff7fffu);
}
__device__ __forceinline__ uint32_t pk_least(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(i16x2, a), __builtin_bit_cast(i16x2, b)));
}
__device__ __forceinline__ uint32_t pk_most(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(i16x2, a), __builtin_bit_cast(i16x2, b)));
}

// Writes the last row_indptr[b + 1] - row_indptr[b] rows of every sequence.  A workgroup
// takes 16 kPass rows of a sequence (a whole number of blocks) for K or V of one head: a
// wave 4 kPass rows in a row, four at a time, all loads first.  Then each wave has the
// bounds of its rows, and the waves of a block join theirs through LDS.
template <int kBits, int kPass, bool kBounds>
__global__ __launch_bounds__(256) void quant_write_kernel(QuantRowsArgs a) {
  constexpr int kRows = 16 * kPass, kWaveRows = 4 * kPass;
  __shared__ __align__(16) uint32_t s_bound[2][16][kHeadDim / 2];  // of the rows of four lane groups of four waves, ordered
  __shared__ uint32_t s_odd[16];                                   // bit g: group g of them has a row of NaN
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, sl = lane & 15, grp = lane >> 4;
  const int g = blockIdx.y >> 1;
  const bool values = blockIdx.y & 1;
  // a sequence of m new rows meets at most m / kRows + 2 pieces of its cache
  const Source src = source_of<kRows, 2>(a, blockIdx.x);
  const int b = src.b;
  const int64_t r0 = src.first, m = src.rows, kvb = src.kvb, n = src.n;
  const int64_t start = max(n - m, (int64_t)0);  // the first row that is written
  const int64_t piece = start / kRows + ((int64_t)blockIdx.x - (r0 / kRows + 2 * (int64_t)b));
  if (m <= 0 || piece * kRows >= n) return;
  const int row0 = (int)(piece * kRows) + wave * kWaveRows + grp;
  // rows before the new ones count for the bounds from the first touched block on
  const int log_block = kBounds ? __builtin_ctz(a.kv.block) : 0;
  const int64_t from = kBounds && !values ? start >> log_block << log_block : start;

  const uint16_t* in = values ? a.v : a.k;
  uint8_t* codes = values ? a.kv.V : a.kv.K;
  uint8_t* scales = values ? a.kv.V_scale : a.kv.K_scale;
  uint4 x[kPass];
  uint2 old[kPass];
  int byte[kPass];
  int64_t place[kPass];
#pragma unroll
  for (int i = 0; i < kPass; ++i) {
    const int row = row0 + 4 * i;
    x[i] = make_uint4(0u, 0u, 0u, 0u);
    if (row >= start && row < n) x[i] = load_stream16(in + ((r0 + row - (n - m)) * a.Hkv + g) * kHeadDim + sl * 8);
  }
#pragma unroll
  for (int i = 0; i < kPass; ++i) {  // (behind the loads: a page's place is one more)
    const int row = row0 + 4 * i;
    place[i] = row >= from && row < n ? place_of(a.kv, a.Hkv, a.total, kvb, b, g, row) : -1;
  }
#pragma unroll
  for (int i = 0; i < kPass; ++i) {
    old[i] = make_uint2(0u, 0u);
    byte[i] = 127;
    if (kBounds && place[i] >= 0 && row0 + 4 * i < start) {
      old[i] = load_codes<kBits>(codes + place[i] * kRowBytes<kBits> + sl * kBits);
      byte[i] = scales[place[i] * 4 + (sl >> 2)];
    }
  }
  uint32_t lo[4], hi[4];  // of two dimensions each
  bool odd = false;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    lo[e] = 0x7fff7fffu;
    hi[e] = 0x80008000u;
  }
#pragma unroll
  for (int i = 0; i < kPass; ++i) {
    const int row = row0 + 4 * i;
    if (row < from || row >= n) continue;
    uint2 c = old[i];
    int s = byte[i];
    if (row >= start) {
      s = scale_byte<kBits>(largest(x[i]));
      c = encode8<kBits>(x[i], s);
      if (place[i] >= 0) {
        uint8_t* to = codes + place[i] * kRowBytes<kBits> + sl * kBits;
        if constexpr (kBits == 8) *reinterpret_cast<uint2*>(to) = c;
        else *reinterpret_cast<uint32_t*>(to) = c.x;
        if ((sl & 3) == 0) scales[place[i] * 4 + (sl >> 2)] = (uint8_t)s;
      } else {  // of a page that is not there: zeros, as they read
        c = make_uint2(0u, 0u);
        s = 127;
      }
    }
    if constexpr (kBounds) {
      if (!values) {
        odd |= s == 255;
        const uint4 d = decode8<kBits>(c, power_of(s));
        const uint32_t w[4] = {ordered(d.x), ordered(d.y), ordered(d.z), ordered(d.w)};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          lo[e] = pk_least(lo[e], w[e]);
          hi[e] = pk_most(hi[e], w[e]);
        }
      }
    }
  }
  if constexpr (kBounds) {
    if (values) return;  // (the whole workgroup)
    *reinterpret_cast<uint4*>(&s_bound[0][wave * 4 + grp][sl * 4]) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    *reinterpret_cast<uint4*>(&s_bound[1][wave * 4 + grp][sl * 4]) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    const uint64_t odd_lanes = __ballot(odd) >> (16 * grp);
    if (sl == 0) s_odd[wave * 4 + grp] = (uint32_t)(odd_lanes & 1) | (uint32_t)(odd_lanes >> 3 & 2) | (uint32_t)(odd_lanes >> 6 & 4) | (uint32_t)(odd_lanes >> 9 & 8);
    __syncthreads();
    // block j of the piece: the lane groups of its rows; a thread takes two dimensions of one side
    if (tid >= kHeadDim) return;
    const int per = 4 * max(1, a.kv.block / kWaveRows), blocks = kRows >> log_block;
    const int64_t out = (int64_t)g * ((a.total >> log_block) + a.B) + first_block(kvb, log_block, b);
    const int side = tid >> 6, d = tid & 63;
    for (int j = 0; j < blocks; ++j) {
      const int64_t block = piece * blocks + j;
      if (block << log_block < from || block << log_block >= n) continue;
      uint32_t v = side ? 0x80008000u : 0x7fff7fffu, bad = 0;
#pragma unroll 4
      for (int w = 0; w < per; ++w) {
        const uint32_t y = s_bound[side][j * per + w][d];
        bad |= s_odd[j * per + w];
        v = side ? pk_most(v, y) : pk_least(v, y);
      }
      // (exact: every value read from the cache is a bf16)
      reinterpret_cast<uint32_t*>(a.kv.bounds)[((out + block) * 2 + side) * (kHeadDim / 2) + d] = bad >> (d >> 4) & 1 ? 0x7fc07fc0u : ordered(v);
    }
  }
}

// Reads the last rows of every sequence, a workgroup 64 of them for K or V of one head;
// rows before a sequence's first are zeros.
template <int kBits>
__global__ __launch_bounds__(256) void quant_read_kernel(QuantRowsArgs a) {
  const int tid = threadIdx.x, sl = tid & 15, sub = tid >> 4;
  const int g = blockIdx.y >> 1;
  const bool values = blockIdx.y & 1;
  const Source src = source_of<64, 1>(a, blockIdx.x);
  const int b = src.b;
  const int64_t r0 = src.first, m = src.rows, kvb = src.kvb, n = src.n;
  const int64_t i0 = ((int64_t)blockIdx.x - (r0 / 64 + b)) * 64;
  const uint8_t* codes = values ? a.kv.V : a.kv.K;
  const uint8_t* scales = values ? a.kv.V_scale : a.kv.K_scale;
  uint16_t* out = (values ? a.V_out : a.K_out) + (int64_t)g * a.n_rows * kHeadDim;
  uint2 c[4];
  int byte[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t at_row = i0 + 16 * i + sub, row = n - m + at_row;
    c[i] = make_uint2(0u, 0u);
    byte[i] = 127;
    if (at_row < m && row >= 0) {
      const int64_t place = place_of(a.kv, a.Hkv, a.total, kvb, b, g, (int)row);
      if (place >= 0) {
        c[i] = load_codes<kBits>(codes + place * kRowBytes<kBits> + sl * kBits);
        byte[i] = scales[place * 4 + (sl >> 2)];
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t at_row = i0 + 16 * i + sub;
    if (at_row < m) store_stream16(out + (r0 + at_row) * kHeadDim + sl * 8, decode8<kBits>(c[i], power_of(byte[i])));
  }
}

template <int kBits>
static void write_t(const QuantRowsArgs& a, hipStream_t st) {
  const int rows = a.kv.bounds && a.kv.block > 64 ? 128 : 64;
  const dim3 grid((uint32_t)(a.n_rows / rows + 2 * (int64_t)a.B), 2 * a.Hkv);
  if (rows == 128) hipLaunchKernelGGL((quant_write_kernel<kBits, 8, true>), grid, dim3(256), 0, st, a);
  else if (a.kv.bounds) hipLaunchKernelGGL((quant_write_kernel<kBits, 4, true>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((quant_write_kernel<kBits, 4, false>), grid, dim3(256), 0, st, a);
}

hipError_t launch_quant_write(const QuantRowsArgs& a, hipStream_t st) {
  if (a.kv.bits == 8) write_t<8>(a, st);
  else write_t<4>(a, st);
  return hipGetLastError();
}

hipError_t launch_quant_read(const QuantRowsArgs& a, hipStream_t st) {
  const dim3 grid((uint32_t)(a.n_rows / 64 + (int64_t)a.B), 2 * a.Hkv);
  if (a.kv.bits == 8) hipLaunchKernelGGL((quant_read_kernel<8>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((quant_read_kernel<4>), grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace tactic
