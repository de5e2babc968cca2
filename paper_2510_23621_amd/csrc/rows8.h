// Rows of 8-bit integers with a scale each.
#pragma once

#include "rows.h"

namespace mace {

constexpr int kMaxColumns8 = 1 << 17;   // 127 * 127 * 2^17 < 2^31: sums of products fit
constexpr int64_t kMaxPitch8 = 1 << 20;       // a tile's rows lie within 32-bit byte offsets
constexpr float kSmallestScale8 = 1.17549435082228751e-38f;   // 2^-126

// Scale of a row whose largest magnitude is m; NaN for an infinite one and for NaN.
// The division is IEEE's, so the scale is the rounded quotient.
__device__ __forceinline__ float scale8(float m) {
  return m < __builtin_inff() ? fmaxf(m / 127.f, kSmallestScale8) : __builtin_nanf("");
}

// The integer nearest to x / s, halves to even, with inv about 1 / s: the product is within
// a hundredth of the quotient, so its nearest integer q is right or off by one next
// to a half, and x - q s is exact (a multiple of half a unit of s, below 2^24 of them, or
// of the smallest number), so that its sign against s / 2 decides.
__device__ __forceinline__ int round8(float x, float s, float inv) {
  float q = rintf(x * inv);
  const float d = __builtin_fmaf(-q, s, x), twice = d + d;
  const bool odd = ((int)q & 1) != 0;
  if (twice > s || (twice == s && odd)) q += 1.f;
  else if (-twice > s || (-twice == s && odd)) q -= 1.f;
  return (int)q;
}
// (inv of a scale next to the smallest is finite; of NaN it is NaN, and the row's values are 0)
__device__ __forceinline__ float inverse8(float s) { return 1.f / s; }

}  // namespace mace
