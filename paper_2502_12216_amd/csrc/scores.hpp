// How attention scores are formed beside the plain dot product: a cap, a bias
// by distance, documents (internal to the library).
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

namespace tactic {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kInvSqrtDim = 0.08838834764831845f;  // 1 / sqrt(128)

// tanh(x) with a relative error near the fp32 rounding everywhere: a cap of 50
// multiplies it, and a weight's relative error is the capped score's absolute one.
// Up to |x| = 1: the continued fraction x / (1 + z / (3 + z / (5 + ... z / 11))),
// z = x^2, as one quotient (cut off there it is off by less than 1e-9).  Beyond:
// 1 - 2 / (1 + e^{2|x|}), which loses nothing to cancellation above 1/2.  NaN stays NaN.
__device__ __forceinline__ float tanh_small(float x) {
  const float z = x * x;
  const float num = fmaf(z, fmaf(z, 21.f, 1260.f), 10395.f);
  const float den = fmaf(z, fmaf(z, z + 210.f, 4725.f), 10395.f);
  return x * num * __builtin_amdgcn_rcpf(den);
}
__device__ __forceinline__ float tanh_large(float x) {
  const float e = __builtin_amdgcn_exp2f(fabsf(x) * (2.f * kLog2e));
  return copysignf(1.f - 2.f * __builtin_amdgcn_rcpf(1.f + e), x);
}
__device__ __forceinline__ float tanh_any(float x) {  // (both, and no branch per lane)
  const float a = tanh_small(x), b = tanh_large(x);
  return fabsf(x) <= 1.f ? a : b;
}

// tanh(x) for |x| <= kTanhPoly: x times the polynomial of degree 5 in x^2 of the least
// largest relative error (by Remez' exchange; with the coefficients in fp32 6.5e-8, with
// fp32 roundings 1.6e-7): seven operations without a reciprocal, for tiles whose scores all lie inside.
constexpr float kTanhPoly = 0.75f;
__device__ __forceinline__ float tanh_poly(float x) {
  const float z = x * x;
  float r = fmaf(z, -0.004716256633400917f, 0.019582906737923622f);
  r = fmaf(z, r, -0.05334442853927612f);
  r = fmaf(z, r, 0.1332540661096573f);
  r = fmaf(z, r, -0.33332958817481995f);
  r = fmaf(z, r, 1.f);
  return x * r;
}

// cap tanh(s / cap) in base 2 for whole tiles of products s = q . k, as s times a
// polynomial in s^2 whose coefficients hold the scale, the cap and log2(e) (set on the
// host in 64 bits): of degree 3 up to |s| = near (a relative error of 6.1e-8 with exact
// arithmetic, 2.2e-7 with fp32's), else of degree 5 up to |s| = far (as tanh_poly).
// near and far are 0.375 and 0.75 of the cap where fp32 holds the coefficients, which go
// with cap^-2j.  Below a cap of 6e-6 (degree 3: 2.5e-8) the last ones are infinite: no |s|
// is inside.  Above 280 (8e4) they are below the normal numbers and count as lost, an
// error of 2^-126 s^2j of the 0.1275 s: within 2^-26 up to |s| = 2^9.5 (2^16).
struct CapPoly {
  float near, far;
  float c3[4], c5[6];
};
__host__ inline CapPoly cap_poly(float cap) {
  CapPoly p{};
  if (!(cap > 0.f)) return p;
  const double c3[4] = {0.9999999403953552, -0.333319753408432, 0.13284501433372498, -0.0482722632586956};
  const double c5[6] = {1.0, -0.33332958817481995, 0.1332540661096573, -0.05334442853927612, 0.019582906737923622,
                        -0.004716256633400917};
  const double k = 0.08838834764831845 / cap, out = cap * 1.4426950408889634;
  double f = k * out;
  for (int i = 0; i < 6; ++i, f *= k * k) {
    if (i < 4) p.c3[i] = (float)(c3[i] * f);
    p.c5[i] = (float)(c5[i] * f);
  }
  const auto limit = [](double by_cap, const float* c, int n, double by_loss) {
    for (int i = 0; i < n; ++i)
      if (!(fabsf(c[i]) < INFINITY)) return -1.f;
    return (float)(fabsf(c[n - 1]) >= 0x1p-126f || by_cap < by_loss ? by_cap : by_loss);
  };
  p.near = limit(0.375 / k, p.c3, 4, 65536.0);
  p.far = limit(0.75 / k, p.c5, 6, 724.0);
  return p;
}
__device__ __forceinline__ float cap_near(float s, const CapPoly& p) {
  const float z = s * s;
  return s * fmaf(z, fmaf(z, fmaf(z, p.c3[3], p.c3[2]), p.c3[1]), p.c3[0]);
}
__device__ __forceinline__ float cap_far(float s, const CapPoly& p) {
  const float z = s * s;
  return s * fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, p.c5[5], p.c5[4]), p.c5[3]), p.c5[2]), p.c5[1]), p.c5[0]);
}

// Score rules of the single-token form (attn_splitk_kernel); every pointer may be null.
struct TokenMod {
  float cap;                    // 0: none
  const float* slopes;          // [Hq]
  const int32_t* positions;     // [Hkv][total] position of each row; null: pos_base[b] + row
  const int32_t* q_pos;         // [B]; null: pos_base[b] + tokens - 1
  const int64_t* pos_base;      // [B] pairs (start, end) of the keys ahead of row 0, their difference is the base; null: 0
  const int32_t* base_of;       // [B] index into pos_base (negative: base 0)
  const int32_t* documents;     // [total] document of each row
  const int32_t* q_documents;   // [B]
  float* scores;                // [Hkv][total][G] base-2 scores out, or null
};
struct NoMod {};

}  // namespace tactic
