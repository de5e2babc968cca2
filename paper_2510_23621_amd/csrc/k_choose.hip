// Choice of experts from a router's logits, and the gradient of the logits:
// mace_choose_forward, mace_choose_backward.
#include <cmath>

#include "rows.h"

namespace mace {
namespace {

constexpr int kMaxChoices = 64, kMaxExpertGroups = 64, kMaxScored = 512;

struct ChooseArgs {
  int64_t n, ld;
  int E, k, groups, top_groups, per;   // per: experts of a group
  int per_inverse;                     // 2^20 / per, rounded up: n per_inverse >> 20 is n / per for n < 512
  int group_lanes;                     // lanes of a group where it is whole lanes, a power of two of them; or 0
  int sigmoid, normalise;
  float scale;
};

template <class T> __device__ __forceinline__ float lowest();
template <> __device__ __forceinline__ float lowest<float>() { return -3.4028234663852886e38f; }
template <> __device__ __forceinline__ float lowest<__bf16>() { return -3.3895313892515355e38f; }
template <> __device__ __forceinline__ float lowest<_Float16>() { return -65504.f; }

// LDS written by some lanes of a wave, read by others: the hardware keeps a wave's order, and this the
// compiler's
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// ------------------------------------------------------------------ lanes of a row
// LPR consecutive lanes hold a token's row. Their sums, maxima and minima go
// through the vector units' own exchanges (DPP, and swaps of half rows), without LDS.
template <int CTRL>
__device__ __forceinline__ int dpp(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true); }
// the two values that a step of distance S joins, in some order: v's and its partner's
template <int S, class X>
__device__ __forceinline__ void exchange(X v, X& a, X& b) {
  constexpr int W = sizeof(X) / 4;
  int in[W], x[W], y[W];
  __builtin_memcpy(in, &v, sizeof(X));
#pragma unroll
  for (int i = 0; i < W; ++i) {
    x[i] = in[i];
    if constexpr (S == 1) y[i] = dpp<0xb1>(in[i]);         // quads as 1 0 3 2
    else if constexpr (S == 2) y[i] = dpp<0x4e>(in[i]);    // quads as 2 3 0 1
    else if constexpr (S == 4) y[i] = dpp<0x141>(in[i]);   // eight lanes mirrored (quads are alike by now)
    else if constexpr (S == 8) y[i] = dpp<0x140>(in[i]);   // sixteen mirrored
    else {
      const auto r = S == 16 ? __builtin_amdgcn_permlane16_swap(in[i], in[i], false, false)
                             : __builtin_amdgcn_permlane32_swap(in[i], in[i], false, false);
      x[i] = r[0], y[i] = r[1];
    }
  }
  __builtin_memcpy(&a, x, sizeof(X));
  __builtin_memcpy(&b, y, sizeof(X));
}
// f over the row's values, in every lane of it (f symmetric in its arguments)
template <int LPR, class X, class F>
__device__ __forceinline__ X over_row(X v, F f) {
  X a, b;
  if constexpr (LPR > 1) exchange<1>(v, a, b), v = f(a, b);
  if constexpr (LPR > 2) exchange<2>(v, a, b), v = f(a, b);
  if constexpr (LPR > 4) exchange<4>(v, a, b), v = f(a, b);
  if constexpr (LPR > 8) exchange<8>(v, a, b), v = f(a, b);
  if constexpr (LPR > 16) exchange<16>(v, a, b), v = f(a, b);
  if constexpr (LPR > 32) exchange<32>(v, a, b), v = f(a, b);
  return v;
}
__device__ __forceinline__ int max_of(int a, int b) { return max(a, b); }
__device__ __forceinline__ float max_of(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ double max_of(double a, double b) { return fmax(a, b); }
__device__ __forceinline__ int min_of(int a, int b) { return min(a, b); }
__device__ __forceinline__ double min_of(double a, double b) { return fmin(a, b); }
template <int LPR, class X>
__device__ __forceinline__ X row_max(X v) { return over_row<LPR>(v, [](X a, X b) { return max_of(a, b); }); }
template <int LPR, class X>
__device__ __forceinline__ X row_sum(X v) { return over_row<LPR>(v, [](X a, X b) { return a + b; }); }
template <int LPR>
__device__ __forceinline__ int row_min(int v) { return over_row<LPR>(v, [](int a, int b) { return min(a, b); }); }
template <int LPR>
__device__ __forceinline__ bool row_any(bool v) { return over_row<LPR>((int)v, [](int a, int b) { return a | b; }); }

// Keys are compared as integers in FP32 (the same order, and maxima that need not quiet a NaN
// first: they fold into the exchange) and as they are in FP64.
constexpr int kNoKey = (int)0xff800000 ^ 0x7fffffff;   // of -infinity
__device__ __forceinline__ int key_of(float v) {   // (of zeros: +0 only)
  const int i = __float_as_int(v);
  return i ^ ((i >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float value_of(int k) { return __int_as_float(k ^ ((k >> 31) & 0x7fffffff)); }
__device__ __forceinline__ double value_of(double k) { return k; }
__device__ __forceinline__ int no_key(int) { return kNoKey; }
__device__ __forceinline__ double no_key(double) { return -__builtin_inff(); }

// exp(-d) and 1 / (1 + exp(-x)); NaN goes through
__device__ __forceinline__ float exp_minus(float d) { return d == d ? exp_neg(fminf(d, 200.f)) : d; }
__device__ __forceinline__ float sigmoid_of(float x) { return x == x ? recip_ge1(1.f + exp_neg(fminf(x, 200.f))) : x; }
// A chosen expert's score over exp(m), m the largest chosen logit (of a sigmoid: at most 0), for
// renormalised weights: no 0 / 0 where all scores underflow
__device__ __forceinline__ float relative_score(float x, float m, bool sigmoid) {
  if (!sigmoid) return exp_minus(m - x);
  return exp_minus(m - (x > 0 ? 0 : x)) / (1 + exp_minus(x > 0 ? x : -x));
}

// V consecutive values of a row, `fill` from `end` on
template <int V, class T>
__device__ __forceinline__ void load_row(const T* p, int first, int end, float fill, float (&x)[V]) {
  if (first + V <= end) {
    typedef T tv __attribute__((ext_vector_type(V)));
    tv t;
    __builtin_memcpy(&t, p + first, sizeof(t));
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = to_f32(t[i]);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = first + i < end ? to_f32(p[first + i]) : fill;
  }
}

// ------------------------------------------------------------------ choice
template <int LPR, int V>
struct ChooseShape {
  static constexpr int ROWS = 256 / LPR;                      // tokens per block
  static constexpr int K = LPR * V < kMaxChoices ? LPR * V : kMaxChoices;
  static constexpr int G = LPR * V < kMaxExpertGroups ? LPR * V : kMaxExpertGroups;
};
template <int LPR, int V>
struct ChooseLds {
  using S = ChooseShape<LPR, V>;
  union {   // of one wave: the waves of a block do not wait for each other
    struct {
      int key[(V + 1) * 64];     // each lane's keys, largest first, and none behind them
      int index[(V + 1) * 64];   // their experts
    } sorted;
    double key[64 / LPR][LPR * V];   // (or integers)
  } wave[4];
  double total[S::ROWS][S::G];   // (or floats)
  int taken[S::ROWS][S::G];
  int index[S::ROWS][S::K];   // the choice
};

// Of a token's keys those outside its top_groups best groups become no_key. True: two groups' totals
// differ by at most tol and a few units of the largest of their parts, which may cancel.
template <class Key, int LPR, int V>
__device__ __forceinline__ bool take_groups(const ChooseArgs& a, Key (&key)[V], float tol, int lane, int row, ChooseLds<LPR, V>& sm) {
  using R = decltype(value_of(Key{}));
  const Key none = no_key(Key{});
  const R empty = -__builtin_inff();   // (total of a group without experts)
  const int first = lane * V;
  R* total = reinterpret_cast<R*>(sm.total[row]);
  bool near_tie = false;
  float part = 0.f;
  auto total_of = [&](Key c1, Key c2) {
    const R v1 = value_of(c1), v2 = value_of(c2);
    if (c1 > none) part = fmaxf(part, fabsf((float)v1));
    if (c2 > none) part = fmaxf(part, fabsf((float)v2));
    return c2 > none ? v1 + v2 : (c1 > none ? v1 : empty);
  };
  auto add_units = [&] { tol = __builtin_fmaf(__int_as_float(row_max<LPR>(__float_as_int(part))), 4.7683716e-7f, tol); };
  // groups before g in the order of their totals, of those from h0 on in steps
  auto better_than = [&](int g, int h0, int step) {
    const R mine = total[g];
    int better = 0;
    for (int h = h0; h < a.groups; h += step) {
      const R o = total[h];
      better += o > mine || (o == mine && h < g);
      near_tie |= h != g && fabsf((float)(o - mine)) <= tol;
    }
    return better;
  };
  // whole lanes: their two best, joined over the group's lanes (eight groups of 32: 54 us where LDS took 64)
  if (a.group_lanes) {
    Key c1 = none, c2 = none;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      c2 = max_of(c2, min_of(c1, key[i]));
      c1 = max_of(c1, key[i]);
    }
    auto over_group = [&](auto join) {
      if (LPR > 1 && a.group_lanes > 1) join(Int<1>{});
      if (LPR > 2 && a.group_lanes > 2) join(Int<2>{});
      if (LPR > 4 && a.group_lanes > 4) join(Int<4>{});
      if (LPR > 8 && a.group_lanes > 8) join(Int<8>{});
      if (LPR > 16 && a.group_lanes > 16) join(Int<16>{});
    };
    over_group([&](auto step) {
      Key a1, b1, a2, b2;
      exchange<decltype(step)::value>(c1, a1, b1);
      exchange<decltype(step)::value>(c2, a2, b2);
      c1 = max_of(a1, b1);
      c2 = max_of(min_of(a1, b1), max_of(a2, b2));
    });
    const int g = min(first * a.per_inverse >> 20, a.groups - 1);
    const R sum = total_of(c1, c2);
    if (first == g * a.per) total[g] = sum;
    add_units();
    wave_sync();
    int better = better_than(g, lane & (a.group_lanes - 1), a.group_lanes);   // the group's lanes share the others
    over_group([&](auto step) {
      int x, y;
      exchange<decltype(step)::value>(better, x, y);
      better = x + y;
    });
    const bool taken = better < a.top_groups;
#pragma unroll
    for (int i = 0; i < V; ++i) key[i] = taken ? key[i] : none;
  } else {
    Key* keys = reinterpret_cast<Key*>(sm.wave[threadIdx.x / 64].key[row % (64 / LPR)]);
#pragma unroll
    for (int i = 0; i < V; ++i) keys[first + i] = key[i];
    wave_sync();
    for (int g = lane; g < a.groups; g += LPR) {
      Key c1 = none, c2 = none;
      for (int j = 0; j < a.per; ++j) {
        const Key c = keys[g * a.per + j];
        c2 = max_of(c2, min_of(c1, c));
        c1 = max_of(c1, c);
      }
      total[g] = total_of(c1, c2);
    }
    add_units();
    wave_sync();
    for (int g = lane; g < a.groups; g += LPR) sm.taken[row][g] = better_than(g, 0, 1) < a.top_groups;
    wave_sync();
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int g = min((first + i) * a.per_inverse >> 20, a.groups - 1);
      key[i] = sm.taken[row][g] ? key[i] : none;
    }
  }
  wave_sync();
  return near_tie;
}

// The choice in FP64, for rows that FP32 cannot decide: k rounds of the largest key with the
// lowest index, stored if `store`.
template <class T, int LPR, int V>
__device__ __noinline__ void choose_exact(ChooseArgs a, const T* logits, const float* bias, double top, int lane, int row,
                                          bool store, ChooseLds<LPR, V>& sm) {
  const double none = -__builtin_inff();
  const int first = lane * V;
  float x[V], b[V];   // (read again: the way here is rare, and the registers of the usual one its own)
  load_row<V>(logits, first, a.E, -__builtin_inff(), x);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    b[i] = 0.f;
    if (!(x[i] > lowest<T>())) x[i] = -__builtin_inff();
  }
  if (bias) load_row<V>(bias, first, a.E, 0.f, b);
  double key[V], sum = 0;
  if (!a.sigmoid) {
#pragma unroll
    for (int i = 0; i < V; ++i) sum += x[i] > none ? exp(x[i] - top) : 0.;
    sum = row_sum<LPR>(sum);
  }
#pragma unroll
  for (int i = 0; i < V; ++i)
    key[i] = x[i] > none ? (a.sigmoid ? 1 / (1 + exp(-(double)x[i])) : exp(x[i] - top) / sum) + b[i] : none;
  if (a.groups > 1) take_groups<double, LPR, V>(a, key, 0.f, lane, row, sm);
  if (!bias)   // the logits decide
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (key[i] > none) key[i] = x[i];
  if (store)
    for (int j = lane; j < a.k; j += LPR) sm.index[row][j] = -1;
  wave_sync();
  for (int j = 0; j < a.k; ++j) {
    double best = key[0];
#pragma unroll
    for (int i = 1; i < V; ++i) best = fmax(best, key[i]);
    best = row_max<LPR>(best);
    const bool on = best > none;
    if (!__any(on)) break;
    int e = 1 << 20;
#pragma unroll
    for (int i = V - 1; i >= 0; --i)
      if (key[i] == best) e = first + i;
    e = row_min<LPR>(e);
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (first + i == e) key[i] = none;
    if (on && store && lane == 0) sm.index[row][j] = e;
  }
  wave_sync();
}

// The choice in FP32. Each lane sorts its keys; a round takes the largest head of the row's
// lanes, of equal ones the first lane's, which holds the lower indices. True: a decision was
// nearer than its error.
//
// Error of a score, in units of 2^-24. Softmax: x - top, its product with the FP32 log2(e) and that constant
// put 2.3 |d| of itself on e = exp(-|d|), d = x - top, and exp2 two: at most 0.9 + 2 of the largest e, which is 1,
// for |d| e^-|d| <= 1 / e. Of the sum of n <= 512 scores that is 2.3 times the mean of |d| weighted with e, at
// most 3.9 (511 experts at |d| = 4.9 beside the best), 2 more, V + 6 for its additions and 2 for the reciprocal: 27.
// Together 30 times M = 1 / sum, the largest score there can be. Sigmoid: 1.3 |x| s (1 - s) <= 0.3
// from the argument, and four from exp2, the sum and the reciprocal, with M = 1. The bound taken, (D + 40) M with D the
// row's largest |d| or |x| up to 100, holds for both with room; infinite arguments (masks, places behind
// the last expert) put D at its end. s + b adds half a unit of itself. Two keys may differ by twice the
// bound, two groups' totals by four times, and by the roundings of two sums.
// b: the bias, -infinity for masked experts.
template <bool SIGMOID, int LPR, int V>
__device__ __forceinline__ bool choose_fast(const ChooseArgs& a, const float (&x)[V], const float (&b)[V], bool biased, float top,
                                            int lane, int row, bool& bad, ChooseLds<LPR, V>& sm) {
  constexpr float kLog2e = 1.44269502162933349609375f;
  int key[V];
  float tol = 0.f;
  bool near_tie = false;
  if (!biased)
#pragma unroll
    for (int i = 0; i < V; ++i) key[i] = key_of(x[i] + 0.f);
  if (biased || a.groups > 1) {   // (otherwise the logits decide, exactly)
    const float base = top > -__builtin_inff() ? top : 0.f;
    float s[V], sum = 0.f;
    int arg = 0;   // of values that are not negative, in the order of their bits
#pragma unroll
    for (int i = 0; i < V; ++i) {   // (masked: the argument is infinite, s 0)
      const float d = SIGMOID ? x[i] : x[i] - base;
      const float e = __builtin_amdgcn_exp2f(d * (SIGMOID ? -kLog2e : kLog2e));
      s[i] = SIGMOID ? __builtin_amdgcn_rcpf(1.f + e) : e;
      sum += s[i];
      arg = max(arg, __float_as_int(fabsf(d)));
    }
    float unit = 1.f;
    if constexpr (!SIGMOID) {
      sum = row_sum<LPR>(sum);
      unit = sum > 0.f ? __builtin_amdgcn_rcpf(sum) : 0.f;   // (nothing but masked experts)
    }
    int scored[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float c = SIGMOID ? s[i] + b[i] : __builtin_fmaf(s[i], unit, b[i]);
      bad |= c != c;
      scored[i] = key_of(c);
    }
    tol = (fminf(__int_as_float(row_max<LPR>(arg)), 100.f) + 40.f) * unit * 1.1920929e-7f + 1e-36f;
    if (a.groups > 1) near_tie = take_groups<int, LPR, V>(a, scored, 2 * tol, lane, row, sm);
#pragma unroll
    for (int i = 0; i < V; ++i)   // (without a bias the logits decide within the groups)
      key[i] = biased ? scored[i] : (scored[i] > kNoKey ? key[i] : kNoKey);
  }
  int index[V];
#pragma unroll
  for (int i = 0; i < V; ++i) index[i] = lane * V + i;
#pragma unroll
  for (int i = 0; i < V; ++i)   // neighbours change places only if the second is larger: equal ones keep their order
#pragma unroll
    for (int j = i & 1; j + 1 < V; j += 2) {
      const int k0 = key[j], k1 = key[j + 1], i0 = index[j], i1 = index[j + 1];
      const bool swap = k1 > k0;
      key[j] = max(k0, k1), key[j + 1] = min(k0, k1);
      index[j] = swap ? i1 : i0, index[j + 1] = swap ? i0 : i1;
    }
  const int wl = threadIdx.x & 63;
  auto& sorted = sm.wave[threadIdx.x / 64].sorted;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    sorted.key[64 * i + wl] = key[i];
    sorted.index[64 * i + wl] = index[i];
  }
  sorted.key[64 * V + wl] = kNoKey;
  for (int j = lane; j < a.k; j += LPR) sm.index[row][j] = -1;
  wave_sync();
  int head = key[0], expert = index[0], at = wl;
  float before = __builtin_inff();
  // the row's lanes below this one
  const unsigned long long below = ((1ull << lane) - 1) << (wl & ~(LPR - 1));
  const int rounds = biased ? a.k + 1 : a.k;   // (one more, to see how near the next one came)
  for (int j = 0; j < rounds; ++j) {
    const int best = row_max<LPR>(head);
    const bool has = head == best && best > kNoKey;
    const unsigned long long m = __ballot(has);
    if (!m) break;
    if (biased) {
      const float v = value_of(best);
      near_tie |= best > kNoKey && before - v <= __builtin_fmaf(fabsf(v), 2.3841858e-7f, tol);
      before = v;
    }
    if (has && !(m & below)) {
      if (j < a.k) sm.index[row][j] = expert;
      at += 64;
      head = sorted.key[at];
      expert = sorted.index[at];
    }
  }
  wave_sync();
  return row_any<LPR>(near_tie);
}

// LPR lanes per token, V consecutive experts each. Scores in FP32; the few rows where a decision lies
// within their error are decided again in FP64 (0.9 % of the rows below, a second pass for 1.8 % of the
// waves, and up to three times as many with masked experts or lanes that the experts do not fill, where the bound of
// the error is at its end; all of it in FP64, the first form, took 254 us). Bound by instructions: 36,864 tokens, 8 of 256
// experts in 4 of 8 groups, 35.2 us, the vector units busy 69 % of it with 810 instructions for two tokens, of which
// the lanes' sorting takes 150, nine rounds 220, scores and masks 200, groups 95, weights 60; the 38 MB of
// logits would take 7.5. 16 lanes of 16 experts take 45 where 32 of 8 take 41, 64 of 4 48; one kernel for both
// scores 41.
template <class T, bool SIGMOID, int LPR, int V>
__global__ void __launch_bounds__(256)
choose_kernel(ChooseArgs a, const T* __restrict__ logits, const float* __restrict__ bias, int* __restrict__ expert,
              float* __restrict__ weights) {
  using S = ChooseShape<LPR, V>;
  __shared__ ChooseLds<LPR, V> sm;
  const int lane = threadIdx.x % LPR, row = threadIdx.x / LPR;
  const int64_t t = (int64_t)block_id() * S::ROWS + row;
  if (t - row >= a.n) return;   // (a grid's last row of blocks is full)
  const bool live = t < a.n;   // (a wave's other rows go on)
  const int64_t at = live ? t : 0;
  const float none = -__builtin_inff();
  float x[V], b[V];
  load_row<V>(logits + at * a.ld, lane * V, a.E, none, x);
#pragma unroll
  for (int i = 0; i < V; ++i) b[i] = 0.f;
  if (bias) load_row<V>(bias, lane * V, a.E, 0.f, b);
  bool bad = false;
  constexpr float largest = SIGMOID ? __builtin_inff() : 3.4028234663852886e38f;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    bad |= !(x[i] <= largest);
    const bool on = x[i] > lowest<T>();
    x[i] = on ? x[i] : none;
    b[i] = on ? b[i] : none;
  }
  float top = none;
  if constexpr (!SIGMOID) {
#pragma unroll
    for (int i = 0; i < V; ++i) top = fmaxf(top, x[i]);
    top = row_max<LPR>(top);
  }
  const bool again = choose_fast<SIGMOID, LPR, V>(a, x, b, bias != nullptr, top, lane, row, bad, sm);
  if (__any(again)) choose_exact<T, LPR, V>(a, logits + at * a.ld, bias, top, lane, row, again, sm);
  bad = row_any<LPR>(bad);
  float norm = 0.f;   // sum of exp(x - top) of the softmax
  if (!SIGMOID && !a.normalise) {
#pragma unroll
    for (int i = 0; i < V; ++i) norm += x[i] > none ? exp_minus(top - x[i]) : 0.f;
    norm = row_sum<LPR>(norm);
  }
  constexpr int P = (S::K + LPR - 1) / LPR;
  float v[P], most = none, total = 0.f;
#pragma unroll
  for (int p = 0; p < P; ++p) {
    if (p * LPR >= a.k) break;
    const int j = lane + p * LPR, e = j < a.k ? sm.index[row][j] : -1;
    v[p] = none;
    if (e >= 0) v[p] = to_f32(logits[at * a.ld + e]);
    most = fmaxf(most, v[p]);
  }
  most = row_max<LPR>(most);
  if (SIGMOID) most = fminf(most, 0.f);
#pragma unroll
  for (int p = 0; p < P; ++p) {
    if (p * LPR >= a.k) break;
    if (!(v[p] > none)) v[p] = 0.f;
    else if (a.normalise) v[p] = relative_score(v[p], most, SIGMOID);
    else v[p] = SIGMOID ? sigmoid_of(v[p]) : exp_minus(top - v[p]) / norm;
    total += v[p];
  }
  total = a.normalise ? row_sum<LPR>(total) : 1.f;
  if (!live) return;
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int j = lane + p * LPR;
    if (j >= a.k) break;
    const int e = sm.index[row][j];
    expert[t * a.k + j] = bad ? j : e;
    weights[t * a.k + j] = bad ? __builtin_nanf("") : (e >= 0 ? a.scale * (v[p] / total) : 0.f);
  }
}

// ------------------------------------------------------------------ gradient
template <int LPR, int V>
struct ChooseGradLds {
  using S = ChooseShape<LPR, V>;
  float d[S::ROWS][LPR * V];
  int place[S::ROWS][LPR * V];
};

// v_j are the (renormalised) scores, g_j the weights' gradients: renormalised
// dlogit_j = scale v_j (g_j - sum g v), times 1 - s_j for a sigmoid; otherwise scale s_j
// g_j, times 1 - s_j or less scale s_e sum g s for every expert e. The chosen experts' values are
// scattered through LDS; only a softmax that is not renormalised reads all logits. 36,864 x 256 FP32, 8
// chosen: 14 us, 38 MB written and 21 read; with a comparison for each expert and choice instead of the
// scatter 37.
template <class T, int LPR, int V>
__global__ void __launch_bounds__(256)
choose_bwd_kernel(ChooseArgs a, const float* __restrict__ dweights, const T* __restrict__ logits,
                  const int* __restrict__ expert, T* __restrict__ dlogits, int64_t ld_d) {
  using S = ChooseShape<LPR, V>;
  __shared__ ChooseGradLds<LPR, V> sm;
  const int lane = threadIdx.x % LPR, row = threadIdx.x / LPR, first = lane * V;
  const int64_t t = (int64_t)block_id() * S::ROWS + row;
  if (t - row >= a.n) return;   // (a grid's last row of blocks is full)
  const bool live = t < a.n;
  const int64_t at = live ? t : 0;
  const float none = -__builtin_inff();
  const bool dense = !a.sigmoid && !a.normalise;
  float x[V], top = none, norm = 0.f;
  if (dense) {
    load_row<V>(logits + at * a.ld, first, a.E, none, x);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (x[i] <= lowest<T>()) x[i] = none;   // (NaN stays)
      top = fmaxf(top, x[i]);
    }
    top = row_max<LPR>(top);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      x[i] = x[i] == none ? 0.f : exp_minus(top - x[i]);
      norm += x[i];
    }
    norm = row_sum<LPR>(norm);
  }
  constexpr int P = (S::K + LPR - 1) / LPR;
  int e[P];
  float g[P], v[P], l[P], most = none, total = 0.f, inner = 0.f;
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int j = lane + p * LPR;
    e[p] = j < a.k ? expert[at * a.k + j] : -1;
    if (e[p] >= a.E) e[p] = -1;
    g[p] = e[p] >= 0 ? dweights[at * a.k + j] : 0.f;
    l[p] = e[p] >= 0 ? to_f32(logits[at * a.ld + e[p]]) : none;
    most = fmaxf(most, l[p]);
  }
  most = row_max<LPR>(most);
  if (a.sigmoid) most = fminf(most, 0.f);
#pragma unroll
  for (int p = 0; p < P; ++p) {
    v[p] = 0.f;
    if (p * LPR >= a.k) continue;
    if (e[p] >= 0) {
      if (a.normalise) v[p] = relative_score(l[p], most, a.sigmoid);
      else v[p] = a.sigmoid ? sigmoid_of(l[p]) : (l[p] <= lowest<T>() ? 0.f : exp_minus(top - l[p]) / norm);
    }
    total += v[p];
  }
  total = a.normalise ? row_sum<LPR>(total) : 1.f;
#pragma unroll
  for (int p = 0; p < P; ++p) {
    if (e[p] >= 0) v[p] /= total;
    inner += g[p] * v[p];
  }
  inner = row_sum<LPR>(inner);
#pragma unroll
  for (int i = 0; i < V; ++i) sm.d[row][first + i] = 0.f;
  wave_sync();
  // an expert named twice gets both terms, in their order: seen by whose mark stayed
  bool twice = false;
#pragma unroll
  for (int p = 0; p < P; ++p)
    if (e[p] >= 0) sm.place[row][e[p]] = lane + p * LPR;
  wave_sync();
#pragma unroll
  for (int p = 0; p < P; ++p) {
    if (e[p] >= 0) twice |= sm.place[row][e[p]] != lane + p * LPR;
    v[p] *= a.normalise ? g[p] - inner : g[p];
    if (a.sigmoid && e[p] >= 0) v[p] *= sigmoid_of(-l[p]);
  }
  if (!__any(twice)) {
#pragma unroll
    for (int p = 0; p < P; ++p)
      if (e[p] >= 0) sm.d[row][e[p]] = v[p];
  } else {
#pragma unroll
    for (int p = 0; p < P; ++p)
      for (int j = 0; j < LPR; ++j) {
        if (lane == j && e[p] >= 0) sm.d[row][e[p]] += v[p];
        wave_sync();
      }
  }
  wave_sync();
  if (!live || first >= a.E) return;
  typedef T tv __attribute__((ext_vector_type(V)));
  tv out;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    float d = sm.d[row][first + i];
    if (dense && x[i] != 0.f) d -= x[i] / norm * inner;
    out[i] = (T)(a.scale * d);
  }
  T* q = dlogits + t * ld_d + first;
  if (first + V <= a.E) {
    __builtin_memcpy(q, &out, sizeof(out));
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (first + i < a.E) q[i] = out[i];
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
// lanes per token and experts per lane
template <class F>
mace_status with_row(int E, F f) {
  if (E <= 16) return f(Int<4>{}, Int<4>{});
  if (E <= 64) return f(Int<16>{}, Int<4>{});
  if (E <= 128) return f(Int<16>{}, Int<8>{});
  if (E <= 256) return f(Int<32>{}, Int<8>{});
  return f(Int<64>{}, Int<8>{});
}
ChooseArgs args_of(const mace_choose_desc& d, int v) {
  const int per = d.n_experts / d.n_groups, lanes = per % v ? 0 : per / v;
  return {d.n_tokens, d.ld_logits, d.n_experts, d.top_k, d.n_groups, d.top_groups, per, ((1 << 20) + per - 1) / per,
          lanes & (lanes - 1) ? 0 : lanes, d.scores == MACE_SCORES_SIGMOID, d.normalise, (float)d.scale};
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
    return with_row(desc->n_experts, [&](auto lpr, auto v) {
      constexpr int LPR = decltype(lpr)::value, V = decltype(v)::value, rows = ChooseShape<LPR, V>::ROWS;
      const ChooseArgs a = args_of(*desc, V);
      auto f = a.sigmoid ? choose_kernel<T, true, LPR, V> : choose_kernel<T, false, LPR, V>;
      f<<<grid_of((a.n + rows - 1) / rows), 256, 0, (hipStream_t)stream>>>(a, (const T*)logits, bias, expert, weights);
      return launched();
    });
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
    return with_row(desc->n_experts, [&](auto lpr, auto v) {
      constexpr int LPR = decltype(lpr)::value, V = decltype(v)::value, rows = ChooseShape<LPR, V>::ROWS;
      const ChooseArgs a = args_of(*desc, V);
      choose_bwd_kernel<T, LPR, V><<<grid_of((a.n + rows - 1) / rows), 256, 0, (hipStream_t)stream>>>(
          a, dweights, (const T*)logits, expert, (T*)dlogits, ld_dlogits);
      return launched();
    });
  });
}
