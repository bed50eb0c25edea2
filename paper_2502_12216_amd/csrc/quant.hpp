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

// Codes of 8 values (words of two bf16) of a group: 8 or 4 bytes.  The product with the
// power is exact, the conversion rounds to nearest, ties to even; values above the largest
// number (where the power is at its limit) are held to it, a group of NaN has codes 0.
template <int kBits>
__device__ __forceinline__ uint2 encode8(const uint4& x, int byte) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  const float inv = byte == 255 ? 0.f : __uint_as_float((uint32_t)(254 - byte) << 23);
  constexpr float kTop = kBits == 8 ? 448.f : 6.f;
  float y[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[2 * i] = bf16lo(w[i]) * inv;
    y[2 * i + 1] = bf16hi(w[i]) * inv;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = byte == 255 ? 0.f : fminf(fmaxf(y[i], -kTop), kTop);
  uint2 c = make_uint2(0u, 0u);
  if constexpr (kBits == 8) {
    c.x = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    c.x = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], (int)c.x, true);
    c.y = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
    c.y = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], (int)c.y, true);
  } else {
    c.x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, y[0], y[1], 1.f, 0);
    c.x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c.x, y[2], y[3], 1.f, 1);
    c.x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c.x, y[4], y[5], 1.f, 2);
    c.x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c.x, y[6], y[7], 1.f, 3);
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
