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

// The sequence of work item `item` where sequence b's items start at at(b), which rises
// with b: 64 of them looked at in one step, a lane each.  Uniform over the workgroup.
template <typename At>
__device__ __forceinline__ int source_of(int64_t item, int B, At at) {
  const int lane = threadIdx.x & (kWave - 1);
  int b = 0;
  for (int b0 = 0; b0 < B; b0 += kWave) {
    const bool before = b0 + lane < B && at(min(b0 + lane, B - 1)) <= item;
    const int n = __popcll(__ballot(before));
    if (n > 0) b = b0 + n - 1;
    if (n < kWave) break;
  }
  return __builtin_amdgcn_readfirstlane(b);
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
  __shared__ float s_lo[4][kHeadDim], s_hi[4][kHeadDim];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, sl = lane & 15, grp = lane >> 4;
  const int g = blockIdx.y >> 1;
  const bool values = blockIdx.y & 1;
  const int64_t item = blockIdx.x;
  // a sequence of m new rows meets at most m / kRows + 2 pieces of its cache
  auto at = [&](int b) { return a.row_indptr[b] / kRows + 2 * (int64_t)b; };
  const int b = source_of(item, a.B, at);
  const int64_t r0 = a.row_indptr[b], m = a.row_indptr[b + 1] - r0, kvb = a.kv_indptr[b];
  const int64_t n = seq_tokens(a.kv_indptr, a.seq_len, b);
  const int64_t start = max(n - m, (int64_t)0);  // the first row that is written
  const int64_t piece = start / kRows + (item - at(b));
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
    for (int e = 0; e < 8; ++e) {
      if (odd) lo[e] = hi[e] = __builtin_nanf("");
#pragma unroll
      for (int d = 16; d <= 32; d *= 2) {
        const float l = __shfl_xor(lo[e], d, 64), h = __shfl_xor(hi[e], d, 64);
        // (NaN stays)
        lo[e] = l != l || lo[e] != lo[e] ? __builtin_nanf("") : fminf(lo[e], l);
        hi[e] = h != h || hi[e] != hi[e] ? __builtin_nanf("") : fmaxf(hi[e], h);
      }
      if (grp == 0) {
        s_lo[wave][sl * 8 + e] = lo[e];
        s_hi[wave][sl * 8 + e] = hi[e];
      }
    }
    __syncthreads();
    // block j of the piece: the waves of its rows; a thread takes one dimension of one side
    const int per = max(1, a.kv.block / kWaveRows), blocks = kRows >> log_block;
    const int64_t out = (int64_t)g * ((a.total >> log_block) + a.B) + first_block(kvb, log_block, b);
    const int side = tid >> 7, d = tid & 127;
    const float(*src)[kHeadDim] = side ? s_hi : s_lo;
    for (int j = 0; j < blocks; ++j) {
      const int64_t block = piece * blocks + j;
      if (block << log_block < from || block << log_block >= n) continue;
      float v = src[j * per][d];
      for (int w = 1; w < per; ++w) {
        const float y = src[j * per + w][d];
        v = v != v || y != y ? __builtin_nanf("") : side ? fmaxf(v, y) : fminf(v, y);
      }
      // exact: every value read from the cache is a bf16
      a.kv.bounds[((out + block) * 2 + side) * kHeadDim + d] = v != v ? (uint16_t)0x7fc0 : (uint16_t)(__float_as_uint(v) >> 16);
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
  const int64_t item = blockIdx.x;
  auto at = [&](int b) { return a.row_indptr[b] / 64 + (int64_t)b; };
  const int b = source_of(item, a.B, at);
  const int64_t r0 = a.row_indptr[b], m = a.row_indptr[b + 1] - r0, kvb = a.kv_indptr[b];
  const int64_t n = seq_tokens(a.kv_indptr, a.seq_len, b), i0 = (item - at(b)) * 64;
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
