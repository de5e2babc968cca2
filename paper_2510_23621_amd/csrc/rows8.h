// Rows of 8-bit integers with a scale each.
#pragma once

#include "rows.h"

namespace mace {

constexpr int kMaxColumns8 = 1 << 17;   // 127 * 127 * 2^17 < 2^31: sums of products fit
constexpr int64_t kMaxPitch8 = 1 << 20;       // a tile's rows lie within 32-bit byte offsets
constexpr float kSmallestScale8 = 1.17549435082228751e-38f;   // 2^-126

constexpr float kLargestScale8 = 2.67938838901875044e+36f;   // 127 of the next number are infinite

// Scale of a row whose largest magnitude is m; NaN for an infinite one and for NaN.
// The division is IEEE's, so the scale is the rounded quotient (of FP32's largest number the one below it).
__device__ __forceinline__ float scale8(float m) {
  return m < __builtin_inff() ? fminf(fmaxf(m / 127.f, kSmallestScale8), kLargestScale8) : __builtin_nanf("");
}

// The integer nearest to x / s, halves to even, with inv about 1 / s. x inv + 1.5 2^23 rounds the
// product, which is within 127 2^-23 of the quotient, to an integer q, held in its lowest
// bits: right, or off by one next to a half. x - q s is exact (a multiple of half a unit of s, below 2^24
// of them, or of the smallest number), so that its size against s / 2 decides; with q odd a half
// counts too (one more in the order of the bits).
constexpr float kRound8 = 12582912.f;
__device__ __forceinline__ unsigned round8(float x, float s, float inv) {
  const float t = __builtin_fmaf(x, inv, kRound8);
  const float d = __builtin_fmaf(kRound8 - t, s, x);
  const unsigned q = __float_as_uint(t), twice = __float_as_uint(fabsf(d) + fabsf(d));
  const int toward = (__float_as_int(d) >> 31) | 1;
  return q + (twice + (q & 1) > __float_as_uint(s) ? toward : 0);
}
// (inv of a scale next to the smallest is finite; of NaN it is NaN, and the row's values are 0)
__device__ __forceinline__ float inverse8(float s) { return 1.f / s; }

// A row's scale as a power of two, with which its integers are exact numbers of T, and the rest, a
// factor in (0.5, 1]. Where no power does (127 of it beyond T's range, one of it below binary16's smallest
// number; NaN too) the scale itself and 1: its products with the integers are rounded to T, and
// what the factor multiplies stays as it is. Rows packed from small binary16 numbers come back as
// those numbers then: weights' gradients of rows of 1e-6 to 1e-7 are off by 0.5 %, with powers below
// 2^-24 by 1.4 to 8 %.
template <class T>
__device__ __forceinline__ void split_scale8(float s, float& power, float& factor) {
  constexpr bool half = __is_same(T, _Float16);
  const int bits = __float_as_int(s), e = (bits >> 23) + ((bits & 0x7fffff) != 0);   // (a scale is positive and normal)
  const bool exact = e <= 127 + (half ? 9 : 121) && e >= (half ? 127 - 24 : 1);
  power = exact ? __int_as_float(e << 23) : s;
  factor = exact ? s / power : 1.f;
}

// columns 16 c .. 16 c + 15 of a row, zeros past the last (AL: there are none)
template <class T>
struct Cols16 {
  Vec8<T> v[2];
  __device__ __forceinline__ float get(int i) const { return v[i >> 3].get(i & 7); }
};
template <class T, bool AL>
__device__ __forceinline__ Cols16<T> load_cols16(const T* row, int c, int cols) {
  Cols16<T> r;
#pragma unroll
  for (int h = 0; h < 2; ++h) r.v[h] = load8_to<T, AL>(row + 16 * c + 8 * h, row + cols);
  return r;
}

// Magnitudes are compared by their bits: the same order, and infinities and NaN above all numbers.
template <class T> struct Magnitude {   // of two 16-bit types at once
  typedef unsigned short u2 __attribute__((ext_vector_type(2)));
  u2 m = {0, 0};
  __device__ __forceinline__ void add(const Cols16<T>& x) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 8; i += 2)
        m = __builtin_elementwise_max(m, u2{(unsigned short)(x.v[h].v[i] & 0x7fff), (unsigned short)(x.v[h].v[i + 1] & 0x7fff)});
  }
  __device__ __forceinline__ unsigned bits() const { return m[0] > m[1] ? m[0] : m[1]; }
  __device__ __forceinline__ static float value(unsigned b) { return to_f32(__builtin_bit_cast(T, (unsigned short)b)); }
};
template <> struct Magnitude<float> {
  unsigned m = 0;
  __device__ __forceinline__ void add(const Cols16<float>& x) {
#pragma unroll
    for (int i = 0; i < 16; ++i) m = max(m, __float_as_uint(fabsf(x.get(i))));
  }
  __device__ __forceinline__ unsigned bits() const { return m; }
  __device__ __forceinline__ static float value(unsigned b) { return __uint_as_float(b); }
};

__device__ __forceinline__ i4 lowest_bytes(const unsigned (&q)[16]) {
  i4 o;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    o[j] = (int)__builtin_amdgcn_perm(__builtin_amdgcn_perm(q[4 * j + 3], q[4 * j + 2], 0x0c0c0400),
                                      __builtin_amdgcn_perm(q[4 * j + 1], q[4 * j], 0x0c0c0400), 0x05040100);
  return o;
}
// Sixteen columns as integers, exactly.
template <class T>
__device__ __forceinline__ i4 round_cols16(const Cols16<T>& x, float s, float inv) {
  unsigned q[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) q[i] = round8(x.get(i), s, inv);
  i4 o = lowest_bytes(q);
  if (s != s) o = i4{0, 0, 0, 0};
  return o;
}
// The same in a third of the instructions, unless one of them comes next to a half: `again` then
// asks for round_cols16 instead (4 % of a wave's 1024 columns).
template <class T>
__device__ __forceinline__ i4 round_most16(const Cols16<T>& x, float s, float inv, bool& again) {
  unsigned q[16];
  float far = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float t = __builtin_fmaf(x.get(i), inv, kRound8);
    q[i] = __float_as_uint(t);
    far = fmaxf(far, fabsf(__builtin_fmaf(x.get(i), inv, kRound8 - t)));
  }
  again |= far > 0.49998f;
  i4 o = lowest_bytes(q);
  if (s != s) o = i4{0, 0, 0, 0};
  return o;
}

}  // namespace mace
