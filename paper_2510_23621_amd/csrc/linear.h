// What the linear layers' kernels share: activations, arguments and the epilogue.
#pragma once

#include "../../include/mace.h"
#include "dense.h"

namespace mace {

// ------------------------------------------------------------------ activations
// Normal distribution: Phi(z), and exp(-z^2 / 2). erfc(x) = t q(t) exp(-x^2), t =
// 1 / (1 + 0.36 x), with q a degree-9 polynomial fitted to a relative error of
// 1.6e-7 (evaluated in FP32) over x >= 0: no cancellation in either tail.
__device__ __forceinline__ float normal_cdf(float z, float& e) {
  const float x = fminf(fabsf(z), 30.f);
  const float t = recip_ge1(__builtin_fmaf(x, 0.36f * 0.70710678118654752f, 1.f));
  e = exp_neg(0.5f * x * x);
  constexpr float q[10] = {0.20310825109481812f, 0.20310771465301514f, 0.1899440586566925f,  0.16391651332378387f,
                           0.12292544543743134f, 0.10651545226573944f, -0.02863478660583496f, 0.14342354238033295f,
                           -0.14196832478046417f, 0.03766215592622757f};
  float p = q[9];
#pragma unroll
  for (int i = 8; i >= 0; --i) p = __builtin_fmaf(p, t, q[i]);
  const float h = 0.5f * t * p * e;   // Phi(-|z|)
  return z > 0.f ? 1.f - h : h;
}
// act(z) = z gate(z)
template <int ACT>
__device__ __forceinline__ float gate(float z) {
  // 1 / (1 + exp(-z)). exp_neg takes -88 at the least, and infinity not at all: above 88
  // it is 1, below -88 (where z times it is under 2^-120) 0; -infinity times that is NaN, as with GELU
  if constexpr (ACT == MACE_ACT_SILU) return z < -88.f ? 0.f : recip_ge1(1.f + exp_neg(fminf(z, 88.f)));
  float e;
  return normal_cdf(z, e);
}
template <int ACT>
__device__ __forceinline__ float activate(float z) {
  return ACT == MACE_ACT_NONE ? z : z * gate<ACT>(z);
}
// act'(z); beyond |z| = 88 the slopes are 0 and 1 to FP32, and z (1 - s) would
// be inf 0 at an infinite z
__device__ __forceinline__ float activation_slope(float z, int act) {
  z = z > 88.f ? 88.f : (z < -88.f ? -88.f : z);   // (keeps NaN)
  if (act == MACE_ACT_SILU) return silu_grad(z);
  float e;
  const float c = normal_cdf(z, e);
  return __builtin_fmaf(0.39894228040143268f * z, e, c);
}

template <class T>
struct LinearArgs {
  const T *x, *w, *bias, *residual;
  T *y, *z;
  const int* offsets;
  int64_t n, ldx, ldy, ldr, ldz;
  int n_in, n_out, groups, act;
};

// rows behind the last group: zeros
template <class T>
__device__ __forceinline__ void zero_rows(T* y, int64_t ld, int rows, int cols, int tid, int nt) {
  for (int i = tid; i < rows * cols; i += nt) y[(int64_t)(i / cols) * ld + i % cols] = (T)0.f;
}

// SiLU's gate for results of 16 bits: v_exp_f32 and v_rcp_f32 as they are, in a third of gate's
// instructions (infinities: as there). The exponent -z log2(e) is off by 1.3 units of 2^-24 of itself (the product's
// rounding and the constant's), which e^-z / (1 + e^-z) <= 1 brings to at most 1.3 |z| 2^-24 of
// the gate; exp2, the sum and the reciprocal add three units of FP32.
__device__ __forceinline__ float gate16(float z) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269502162933349609375f));
}
template <int ACT, bool FAST>
__device__ __forceinline__ float gate_as(float z) {
  if constexpr (FAST && ACT == MACE_ACT_SILU) return gate16(z);
  return gate<ACT>(z);
}
template <int ACT, bool FAST>
__device__ __forceinline__ float activate_as(float z) {
  return ACT == MACE_ACT_NONE ? z : z * gate_as<ACT, FAST>(z);
}
// act(z) + r: the last product and the sum are one operation wherever they stand
template <int ACT, bool FAST>
__device__ __forceinline__ float activate_add(float z, float r) {
  return ACT == MACE_ACT_NONE ? z + r : __builtin_fmaf(z, gate_as<ACT, FAST>(z), r);
}

// The epilogue of a block's product: y = act(value + b) + r, z = value + b where it is
// wanted, of the run's rows and the columns from c0 on (y and z point there).
// value(j, i, b): the product at vector j of tile row i, as lane_values orders them, and b.
// AHEAD tile rows of residuals are requested before the first is used, FAST: gate16.
template <class T, bool AL, class S, int AHEAD = 1, bool FAST = false, class F>
__device__ __forceinline__ void linear_epilogue(const LinearArgs<T>& a, const RowRun& run, int c0, int cols, T* y, T* z,
                                                int tid, F value) {
  constexpr int W = lane_width<T>, NV = lane_vectors<S::TN, W>, RING = AHEAD + 1 < S::TM ? AHEAD + 1 : S::TM;
  using V = typename Floats<W>::type;
  typedef T tw __attribute__((ext_vector_type(W)));
  const int l = tid & 63, wv = tid >> 6;
  const int m0 = (wv / S::WN) * (S::BM / S::WM) + (l & 15), n0 = (wv % S::WN) * (S::BN / S::WN);
  const T* bias = a.bias ? a.bias + (int64_t)run.group * a.n_out + c0 : nullptr;
  const T* res = a.residual ? a.residual + run.row0 * a.ldr + c0 : nullptr;
  auto finish = [&](auto act) {
    V bj[NV];
    tw rj[RING][NV];   // (as they lie in memory: half the registers of 16-bit types)
    auto column = [&](int j) { return n0 + lane_column<W>(j, l); };
    auto count = [&](int j) { return AL ? W : min(W, cols - column(j)); };
    auto load_residual = [&](int i) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (m0 + 16 * i < run.rows && column(j) < cols)
          rj[i % RING][j] = read_raw<W>(res + (int64_t)(m0 + 16 * i) * a.ldr + column(j), count(j), AL);
    };
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      bj[j] = V{};
      if (bias && column(j) < cols) bj[j] = read_n<W>(bias + column(j), count(j), AL);
    }
    if (res)
#pragma unroll
      for (int i = 0; i < RING - 1; ++i) load_residual(i);
#pragma unroll
    for (int i = 0; i < S::TM; ++i) {
      const int64_t m = m0 + 16 * i;
      if (res && i + RING - 1 < S::TM) load_residual(i + RING - 1);
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        V v = value(j, i, bj[j]);
        const int n = column(j);
        if (m >= run.rows || n >= cols) continue;
        if (z) store_n(z + m * a.ldz + n, v, count(j), AL);
        constexpr int ACT = decltype(act)::value;
        if (res) {
#pragma unroll
          for (int q = 0; q < W; ++q) v[q] = activate_add<ACT, FAST>(v[q], (float)rj[i % RING][j][q]);
        } else {
#pragma unroll
          for (int q = 0; q < W; ++q) v[q] = activate_as<ACT, FAST>(v[q]);
        }
        store_n(y + m * a.ldy + n, v, count(j), AL);
      }
    }
  };
  if (a.act == MACE_ACT_SILU) finish(Int<MACE_ACT_SILU>{});
  else if (a.act == MACE_ACT_GELU) finish(Int<MACE_ACT_GELU>{});
  else finish(Int<MACE_ACT_NONE>{});
}

}  // namespace mace
