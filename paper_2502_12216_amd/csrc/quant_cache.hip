// Rows into a cache of 8 or 4 bits, with the bounds of their blocks, and out of it.
//
// Both move bytes: a row of K or V is 256 bytes in bf16 and 132 or 68 in the cache.  16
// lanes share a row, 8 values each, so that a group of 32 is four lanes and its largest
// value two DPP steps; nothing is read twice but the rows of a block that was begun
// before, whose bounds are taken again from the cache.
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
  const int64_t page = kv.pk.page_table[(int64_t)b * kv.pk.max_pages + min(row / kv.pk.page_size, kv.pk.max_pages - 1)];
  if (page < 0 || page >= kv.pk.num_pages) return -1;
  return (page * Hkv + g) * kv.pk.page_size + row % kv.pk.page_size;
}

template <int kBits>
__device__ __forceinline__ uint2 load_codes(const uint8_t* p) {
  if constexpr (kBits == 8) return *reinterpret_cast<const uint2*>(p);
  else return make_uint2(*reinterpret_cast<const uint32_t*>(p), 0u);
}

__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false));
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false));
}

// Writes the last row_indptr[b + 1] - row_indptr[b] rows of every sequence.  A workgroup
// takes 16 kPass rows of a sequence (a whole number of blocks) for K or V of one head: a
// wave 4 kPass rows in a row, four at a time, all loads first.  Then each wave has the
// bounds of its rows, and the waves of a block join theirs through LDS.
template <int kBits, int kPass, bool kBounds>
__global__ __launch_bounds__(256) void quant_write_kernel(QuantRowsArgs a) {
  constexpr int kRows = 16 * kPass, kWaveRows = 4 * kPass;
  __shared__ __align__(16) float s_bound[2][16][kHeadDim];  // of the rows of four lane groups of four waves
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
    place[i] = -1;
    x[i] = make_uint4(0u, 0u, 0u, 0u);
    old[i] = make_uint2(0u, 0u);
    byte[i] = 127;
    if (row >= from && row < n) place[i] = place_of(a.kv, a.Hkv, a.total, kvb, b, g, row);
    if (row >= start && row < n) x[i] = load_stream16(in + ((r0 + row - (n - m)) * a.Hkv + g) * kHeadDim + sl * 8);
  }
  if constexpr (kBounds) {
#pragma unroll
    for (int i = 0; i < kPass; ++i) {
      if (place[i] >= 0 && row0 + 4 * i < start) {
        old[i] = load_codes<kBits>(codes + place[i] * kRowBytes<kBits> + sl * kBits);
        byte[i] = scales[place[i] * 4 + (sl >> 2)];
      }
    }
  }
  float lo[8], hi[8];
  bool odd = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    lo[e] = INFINITY;
    hi[e] = -INFINITY;
  }
#pragma unroll
  for (int i = 0; i < kPass; ++i) {
    const int row = row0 + 4 * i;
    if (row < from || row >= n) continue;
    uint2 c = old[i];
    int s = byte[i];
    if (row >= start) {
      uint32_t top = 0;
      const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) top = max(top, max(w[e] & 0x7fffu, (w[e] >> 16) & 0x7fffu));
      s = scale_byte<kBits>(quad_max(top));
      c = encode8<kBits>(x[i], s);
      if (place[i] >= 0) {
        uint8_t* to = codes + place[i] * kRowBytes<kBits> + sl * kBits;
        if constexpr (kBits == 8) *reinterpret_cast<uint2*>(to) = c;
        else *reinterpret_cast<uint32_t*>(to) = c.x;
        if ((sl & 3) == 0) scales[place[i] * 4 + (sl >> 2)] = (uint8_t)s;
      }
    }
    if constexpr (kBounds) {
      if (!values) {
        odd |= s == 255;
        const uint4 d = decode8<kBits>(c, power_of(s));
        const uint32_t w[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          lo[2 * e] = fminf(lo[2 * e], bf16lo(w[e]));
          hi[2 * e] = fmaxf(hi[2 * e], bf16lo(w[e]));
          lo[2 * e + 1] = fminf(lo[2 * e + 1], bf16hi(w[e]));
          hi[2 * e + 1] = fmaxf(hi[2 * e + 1], bf16hi(w[e]));
        }
      }
    }
  }
  if constexpr (kBounds) {
    if (values) return;  // (the whole workgroup)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (odd) lo[e] = hi[e] = __builtin_nanf("");
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
      *reinterpret_cast<float4*>(&s_bound[0][wave * 4 + grp][sl * 8 + e]) = make_float4(lo[e], lo[e + 1], lo[e + 2], lo[e + 3]);
      *reinterpret_cast<float4*>(&s_bound[1][wave * 4 + grp][sl * 8 + e]) = make_float4(hi[e], hi[e + 1], hi[e + 2], hi[e + 3]);
    }
    __syncthreads();
    // block j of the piece: the waves of its rows; a thread takes one dimension of one side
    const int per = 4 * max(1, a.kv.block / kWaveRows), blocks = kRows >> log_block;
    const int64_t out = (int64_t)g * ((a.total >> log_block) + a.B) + first_block(kvb, log_block, b);
    const int side = tid >> 7, d = tid & 127;
    for (int j = 0; j < blocks; ++j) {
      const int64_t block = piece * blocks + j;
      if (block << log_block < from || block << log_block >= n) continue;
      float v = side ? -INFINITY : INFINITY;
      bool odd_here = false;
      for (int w = 0; w < per; ++w) {
        const float y = s_bound[side][j * per + w][d];
        odd_here |= y != y;
        v = side ? fmaxf(v, y) : fminf(v, y);
      }
      // exact: every value read from the cache is a bf16
      a.kv.bounds[((out + block) * 2 + side) * kHeadDim + d] = odd_here ? (uint16_t)0x7fc0 : (uint16_t)(__float_as_uint(v) >> 16);
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
