// The format of the quantised cache (internal to the library).
//
// A row of 128 values is four groups of 32 with a power of two each, a byte s + 127
// (255: the group held a value that is not finite, and reads as NaN).  8 bits are e4m3
// (largest 448 = 1.75 2^8, smallest 2^-9), 4 bits e2m1 (6 = 1.5 2^2, 1/2), the first of
// two values in the lower half of the byte.  s is the least power whose largest number
// is not below the group's, kept where every number of the group is a normal bf16 or 0
// ([-117, 119] and [-125, 125]); so each value read is a bf16 exactly.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.hpp"
#include "kernels.hpp"

namespace tactic {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short i16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

template <int kBits>
constexpr int kRowBytes = 16 * kBits;

// The byte of a group from the bits of its largest |bf16| (which order as the values do)
template <int kBits>
__device__ __forceinline__ int scale_byte(uint32_t top) {
  if (top >= 0x7f80u) return 255;
  const int e = (int)(top >> 7), m = (int)(top & 127u);
  return kBits == 8 ? min(max(e - 8 + (m > 96), 10), 246) : min(max(e - 2 + (m > 64), 2), 252);
}
__device__ __forceinline__ float power_of(int byte) { return __uint_as_float((uint32_t)byte << 23); }  // (255: inf, makes NaN of any code)

// Codes of 8 values (words of two bf16) of a group: 8 or 4 bytes.  The conversions divide by the power
// and round to nearest, ties to even (checked for every bf16).  Values above the largest number
// (where the power is at its limit) are held to it: e2m1's conversion does, e4m3's gives NaN
// beyond 464.  A group of NaN has codes 0.
template <int kBits>
__device__ __forceinline__ uint2 encode8(const uint4& x, int byte) {
  uint32_t w[4] = {x.x, x.y, x.z, x.w};
  const uint32_t keep = byte == 255 ? 0u : ~0u;
  const float power = power_of(byte == 255 ? 127 : byte);
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] &= keep;
  if (kBits == 8 && __any(byte == 246)) {
    constexpr uint32_t kTop = 0x7f60u;  // 448 2^119
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = min(w[i] & 0x7fffu, kTop), hi = min(w[i] >> 16 & 0x7fffu, kTop);
      if (byte == 246) w[i] = (w[i] & 0x80008000u) | hi << 16 | lo;
    }
  }
  uint2 c = make_uint2(0u, 0u);
  if constexpr (kBits == 8) {
    i16x2 lo = {0, 0}, hi = {0, 0};
    lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, __builtin_bit_cast(bf16x2, w[0]), power, false);
    lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, __builtin_bit_cast(bf16x2, w[1]), power, true);
    hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, __builtin_bit_cast(bf16x2, w[2]), power, false);
    hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, __builtin_bit_cast(bf16x2, w[3]), power, true);
    c = make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
  } else {
    c.x = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, __builtin_bit_cast(bf16x2, w[0]), power, 0);
    c.x = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c.x, __builtin_bit_cast(bf16x2, w[1]), power, 1);
    c.x = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c.x, __builtin_bit_cast(bf16x2, w[2]), power, 2);
    c.x = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c.x, __builtin_bit_cast(bf16x2, w[3]), power, 3);
  }
  return c;
}

// The pair of values p (a constant after unrolling) of a word of codes, as two bf16:
// pairs 0 and 1 of 8 bits, 0 to 3 of 4 bits
template <int kBits>
__device__ __forceinline__ uint32_t decode_pair(uint32_t w, int p, float power) {
  if constexpr (kBits == 8) {
    return p == 0 ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, power, false))
                  : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, power, true));
  } else {
    switch (p) {
      case 0: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, power, 0));
      case 1: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, power, 1));
      case 2: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, power, 2));
      default: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, power, 3));
    }
  }
}

// 8 values of the codes of encode8, as words of two bf16
template <int kBits>
__device__ __forceinline__ uint4 decode8(const uint2& c, float power) {
  if constexpr (kBits == 8)
    return make_uint4(decode_pair<8>(c.x, 0, power), decode_pair<8>(c.x, 1, power), decode_pair<8>(c.y, 0, power), decode_pair<8>(c.y, 1, power));
  else
    return make_uint4(decode_pair<4>(c.x, 0, power), decode_pair<4>(c.x, 1, power), decode_pair<4>(c.x, 2, power), decode_pair<4>(c.x, 3, power));
}

// First place of sequence b's blocks in the bounds: spans do not overlap, since
// floor((x + y) / L) - floor(x / L) + 1 >= ceil(y / L)
// (L = 2^log_block)
__device__ __forceinline__ int64_t first_block(int64_t kvb, int log_block, int b) { return (kvb >> log_block) + b; }

}  // namespace tactic
