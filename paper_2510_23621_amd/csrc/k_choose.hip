// Choice of experts from a router's logits, and the gradient of the logits:
// mace_choose_forward, mace_choose_backward.
#include <cmath>

#include "rows.h"

namespace mace {
namespace {

constexpr int kMaxChoices = 64, kMaxExpertGroups = 64, kMaxScored = 512;
constexpr int kPerLane = kMaxScored / 64;

struct ChooseArgs {
  int64_t n, ld;
  int E, k, groups, top_groups, per;   // per: experts of a group
  int sigmoid, normalise;
  float scale;
};

template <class T> __device__ __forceinline__ float lowest();
template <> __device__ __forceinline__ float lowest<float>() { return -3.4028234663852886e38f; }
template <> __device__ __forceinline__ float lowest<__bf16>() { return -3.3895313892515355e38f; }
template <> __device__ __forceinline__ float lowest<_Float16>() { return -65504.f; }

__device__ __forceinline__ double shfl_xor(double v, int m) { return __shfl_xor(v, m); }

// Largest (value, lowest index) over the wave, in every lane; NaN does not occur
__device__ __forceinline__ void wave_best(double& v, int& i) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const double ov = __shfl_xor(v, d);
    const int oi = __shfl_xor(i, d);
    if (ov > v || (ov == v && oi < i)) v = ov, i = oi;
  }
}

// log of 1 / (1 + exp(-l))
__device__ __forceinline__ double log_sigmoid(double l) { return (l < 0 ? l : 0.) - log1p(exp(-fabs(l))); }

// A wave per token, lane l holding experts l, l + 64, ...; all in FP64, so that the order
// of nearly equal scores is that of the scores and not of their roundings.
template <class T>
__global__ void __launch_bounds__(256)
choose_kernel(ChooseArgs a, const T* __restrict__ logits, const float* __restrict__ bias, int* __restrict__ expert,
              float* __restrict__ weights) {
  __shared__ double sm[4][kMaxScored];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t t = (int64_t)block_id() * 4 + w;
  if (t >= a.n) return;
  const double none = -__builtin_inf();
  double l[kPerLane], key[kPerLane];
  double top = none, sum = 0;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) {
    const int e = lane + 64 * i;
    l[i] = none;
    if (e < a.E) {
      const float x = to_f32(logits[t * a.ld + e]);
      bad |= x != x || (!a.sigmoid && x == __builtin_inff());
      if (x > lowest<T>()) l[i] = x;
    }
    top = fmax(top, l[i]);
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = fmax(top, __shfl_xor(top, d));
  double norm = 0;   // log of the softmax's denominator
  if (!a.sigmoid && top > none) {
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) sum += l[i] > none ? exp(l[i] - top) : 0.;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
    norm = top + log(sum);
  }
  // scores
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) {
    const int e = lane + 64 * i;
    double c = none;
    if (l[i] > none) {
      const double s = a.sigmoid ? 1 / (1 + exp(-l[i])) : exp(l[i] - top) / sum;
      c = s + (bias ? (double)bias[e] : 0.);
      bad |= c != c;
    }
    key[i] = c;
    if (e < a.E) sm[w][e] = c;
  }
  __builtin_amdgcn_wave_barrier();
  const bool no_order = __any(bad);
  if (a.groups > 1) {
    double total = none;   // lane g: group g
    if (lane < a.groups) {
      double c1 = none, c2 = none;
      for (int j = 0; j < a.per; ++j) {
        const double c = sm[w][lane * a.per + j];
        if (c > c1) c2 = c1, c1 = c;
        else if (c > c2) c2 = c;
      }
      total = c2 > none ? c1 + c2 : c1;
    }
    unsigned long long taken = 0;
    for (int j = 0; j < a.top_groups; ++j) {
      double v = total;
      int g = lane;
      wave_best(v, g);
      if (!(v > none)) break;
      taken |= 1ull << g;
      if (lane == g) total = none;
    }
#pragma unroll
    for (int i = 0; i < kPerLane; ++i)
      if (!(taken >> ((lane + 64 * i) / a.per) & 1)) key[i] = none;
  }
  if (!bias) {
#pragma unroll
    for (int i = 0; i < kPerLane; ++i)
      if (key[i] > none) key[i] = l[i];
  }
  // lane j keeps choice j
  int chosen = -1;
  double log_score = none;
  for (int j = 0; j < a.k; ++j) {
    double v = none;
    int e = 1 << 20;
#pragma unroll
    for (int i = 0; i < kPerLane; ++i)
      if (key[i] > v) v = key[i], e = lane + 64 * i;
    wave_best(v, e);
    if (!(v > none)) break;
    double mine = 0;
#pragma unroll
    for (int i = 0; i < kPerLane; ++i)
      if (e == lane + 64 * i) key[i] = none, mine = l[i];
    mine = __shfl(mine, e & 63);
    if (lane == j) {
      chosen = e;
      log_score = a.sigmoid ? log_sigmoid(mine) : mine - norm;
    }
  }
  double value = chosen >= 0 ? exp(log_score) : 0.;
  if (a.normalise) {
    double m = log_score;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) m = fmax(m, __shfl_xor(m, d));
    value = chosen >= 0 ? exp(log_score - m) : 0.;
    double total = value;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) total += __shfl_xor(total, d);
    if (chosen >= 0) value /= total;
  }
  if (lane < a.k) {
    expert[t * a.k + lane] = no_order ? lane : chosen;
    weights[t * a.k + lane] = no_order ? __builtin_nanf("") : (float)(a.scale * value);
  }
}

// A wave per token. v_j are the (renormalised) scores, g_j the weights' gradients:
// renormalised dlogit_j = scale v_j (g_j - sum g v), times 1 - s_j for a sigmoid;
// otherwise scale s_j g_j, times 1 - s_j or less scale s_e sum g s for every expert e.
template <class T>
__global__ void __launch_bounds__(256)
choose_bwd_kernel(ChooseArgs a, const float* __restrict__ dweights, const T* __restrict__ logits,
                  const int* __restrict__ expert, T* __restrict__ dlogits, int64_t ld_d) {
  const int lane = threadIdx.x & 63;
  const int64_t t = (int64_t)block_id() * 4 + (threadIdx.x >> 6);
  if (t >= a.n) return;
  const float none = -__builtin_inff();
  float l[kPerLane], top = none, sum = 0.f;
  const bool dense = !a.sigmoid && !a.normalise;
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) {
    const int e = lane + 64 * i;
    l[i] = e < a.E ? to_f32(logits[t * a.ld + e]) : none;
    if (l[i] <= lowest<T>()) l[i] = none;
    top = fmaxf(top, l[i]);
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
  if (!(top > none)) top = 0.f;
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) sum += expf(l[i] - top);   // (-infinity: 0; NaN goes on)
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
  // lane j: choice j
  int e = -1;
  float x = none, g = 0.f;
  if (lane < a.k) {
    e = expert[t * a.k + lane];
    if (e < 0 || e >= a.E) e = -1;
    if (e >= 0) {
      x = to_f32(logits[t * a.ld + e]);
      g = dweights[t * a.k + lane];
    }
  }
  float s = e < 0 ? 0.f : (a.sigmoid ? 1.f / (1.f + expf(-x)) : expf(x - top) / sum), v = s;
  if (a.normalise) {
    const float ls = e < 0 ? none : (a.sigmoid ? fminf(x, 0.f) - log1pf(expf(-fabsf(x))) : x);
    float m = ls;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
    v = e < 0 ? 0.f : expf(ls - m);
    float total = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) total += __shfl_xor(total, d);
    if (e >= 0) v /= total;
  }
  float inner = g * v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) inner += __shfl_xor(inner, d);
  float mine = a.normalise ? v * (g - inner) : v * g;
  if (a.sigmoid) mine *= 1.f / (1.f + expf(x));
  if (e < 0) mine = 0.f;
  float out[kPerLane] = {};
  for (int j = 0; j < a.k; ++j) {
    const int ej = __shfl(e, j);
    const float dj = __shfl(mine, j);
#pragma unroll
    for (int i = 0; i < kPerLane; ++i)
      if (ej == lane + 64 * i) out[i] += dj;
  }
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) {
    if (dense && l[i] > none) out[i] -= expf(l[i] - top) / sum * inner;
    if (lane + 64 * i < a.E) dlogits[t * ld_d + lane + 64 * i] = (T)(a.scale * out[i]);
  }
}

// ------------------------------------------------------------------ host
mace_status check(const mace_choose_desc* d) {
  if (!d || d->n_tokens < 0 || d->n_experts < 1 || d->top_k < 1 || d->n_groups < 1 || d->top_groups < 1) return MACE_EINVAL;
  if (d->dtype < MACE_TYPE_FP32 || d->dtype > MACE_TYPE_FP16 || (d->normalise & ~1)) return MACE_EINVAL;
  if (d->scores != MACE_SCORES_SOFTMAX && d->scores != MACE_SCORES_SIGMOID) return MACE_EINVAL;
  if (d->n_experts % d->n_groups || d->top_groups > d->n_groups || d->ld_logits < d->n_experts) return MACE_EINVAL;
  if (d->top_k > (int64_t)d->top_groups * (d->n_experts / d->n_groups) || !std::isfinite((float)d->scale)) return MACE_EINVAL;
  if (d->n_experts > kMaxScored || d->n_groups > kMaxExpertGroups || d->top_k > kMaxChoices) return MACE_EUNSUPPORTED;
  if (d->n_tokens > (1 << 30) || d->n_tokens * d->top_k > (1 << 30)) return MACE_EUNSUPPORTED;
  return MACE_OK;
}
ChooseArgs args_of(const mace_choose_desc& d) {
  return {d.n_tokens, d.ld_logits, d.n_experts, d.top_k, d.n_groups, d.top_groups, d.n_experts / d.n_groups,
          d.scores == MACE_SCORES_SIGMOID, d.normalise, (float)d.scale};
}

}  // namespace
}  // namespace mace

using namespace mace;

extern "C" mace_status mace_choose_forward(const mace_choose_desc* desc, const void* logits, const float* bias,
                                           int32_t* expert, float* weights, void* stream) {
  const mace_status st = check(desc);
  if (st != MACE_OK) return st;
  if (desc->n_tokens == 0) return MACE_OK;
  if (!logits || !expert || !weights) return MACE_EINVAL;
  return by_type(desc->dtype, [&](auto zero) -> mace_status {
    using T = decltype(zero);
    const ChooseArgs a = args_of(*desc);
    choose_kernel<T><<<grid_of((a.n + 3) / 4), 256, 0, (hipStream_t)stream>>>(a, (const T*)logits, bias, expert, weights);
    return launched();
  });
}

extern "C" mace_status mace_choose_backward(const mace_choose_desc* desc, const float* dweights, const void* logits,
                                            const int32_t* expert, void* dlogits, int64_t ld_dlogits, void* stream) {
  const mace_status st = check(desc);
  if (st != MACE_OK) return st;
  if (ld_dlogits < desc->n_experts) return MACE_EINVAL;
  if (desc->n_tokens == 0) return MACE_OK;
  if (!dweights || !logits || !expert || !dlogits) return MACE_EINVAL;
  return by_type(desc->dtype, [&](auto zero) -> mace_status {
    using T = decltype(zero);
    const ChooseArgs a = args_of(*desc);
    choose_bwd_kernel<T><<<grid_of((a.n + 3) / 4), 256, 0, (hipStream_t)stream>>>(a, dweights, (const T*)logits, expert,
                                                                                 (T*)dlogits, ld_dlogits);
    return launched();
  });
}
