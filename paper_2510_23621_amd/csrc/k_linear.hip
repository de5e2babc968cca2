// Grouped dense layer y = act(x W_g + b_g) + r and its backward pass:
// mace_linear_forward, mace_linear_backward, mace_linear_backward8.
#include <algorithm>
#include <cmath>

#include "linear.h"
#include "rows8.h"

namespace mace {
namespace {

// ------------------------------------------------------------------ arguments
template <class T>
struct RowGradArgs {
  const T *dz, *w;
  T* dx;
  const int* offsets;
  int64_t n, lddz, lddx;
  int n_in, n_out, groups;
  const float* x_scales;   // of an 8-bit input, or NULL: dz has split_scale8's factors on its rows
};
// dx of row r from its product with dz
template <class T, class V>
__device__ __forceinline__ V without_factor(const RowGradArgs<T>& a, int64_t r, V v) {
  if constexpr (sizeof(T) == 2)
    if (a.x_scales) {
      float power, factor;
      split_scale8<T>(a.x_scales[r], power, factor);
      v *= 1.f / factor;
    }
  return v;
}
template <class T>
struct WeightGradArgs {
  const T *x, *dz;
  T* dw;
  float* part;   // [splits][G][n_in][n_out], or NULL for one split
  const int* offsets;
  int64_t n, ldx, lddz;
  int n_in, n_out, groups, splits;
};
template <class T>
struct BiasGradArgs {
  const float* sums;
  T* db;
  const int* offsets;
  int64_t n;
  int n_out, groups, run_rows, max_runs;
};

// The block's product, by the way its shape and operands allow
template <class T, class S, bool KCR, bool KCC, bool AL>
__device__ __forceinline__ void product(const Operand<T>& ro, const Operand<T>& co, int K, unsigned short* lds, int tid,
                                        f4 (&acc)[S::TN][S::TM]) {
  if constexpr (AL && S::DIRECT) {
    tile_gemm_direct<T, S, KCR, KCC>(ro, co, K, lds, tid, acc);
  } else {
    TileSource<T, S::BM, S::BK, KCR, AL, S::NT, S::DEPTH> r;
    TileSource<T, S::BN, S::BK, KCC, AL, S::NT, S::DEPTH> c;
    r.init(ro.p, ro.ld, ro.rows, tid, ro.end);
    c.init(co.p, co.ld, co.rows, tid, co.end);
    tile_gemm<T, S, KCR, KCC, AL>(r, c, K, lds, tid, acc);
  }
}

// FP32 launches of few tiles: a block of four waves forms 16 RT x 16 CT results on
// FP32 MFMA (v_mfma_f32_16x16x4: no splitting, and with few rows the weights' way
// from memory bounds it, not the products), each wave every fourth run of 32 k;
// the four partial sums are added through LDS. Lane l takes k + 8 (l/16) + 0..7 of
// operand row l%16, straight from memory, a step ahead. f(row, column, values, count).
template <int RT_, int CT_> struct ThinShape {
  static constexpr int RT = RT_, CT = CT_, BM = 16 * RT, BN = 16 * CT, NT = 256;
};
template <class S, bool KCC, bool AL, class F>
__device__ __forceinline__ void thin_product(const Operand<float>& ro, const Operand<float>& co, int K, float* lds, int tid,
                                             F f) {
  constexpr int RT = S::RT, CT = S::CT;
  const int l = tid & 63, wv = tid >> 6, i = l & 15, g = l >> 4;
  const float *x[RT], *w[CT];
#pragma unroll
  for (int r = 0; r < RT; ++r) x[r] = ro.p + min(16 * r + i, ro.rows - 1) * ro.ld + 8 * g;
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const int64_t n = min(16 * c + i, co.rows - 1);
    w[c] = co.p + (KCC ? n * co.ld + 8 * g : n + 8 * g * co.ld);
  }
  Vec8<float> xv[2][RT], wv8[2][CT];
  auto load = [&](auto d_, int k) {
    constexpr int D = decltype(d_)::value;
    const int n = K - k - 8 * g;   // this lane's k in bounds
    const bool whole = k + 32 <= K;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      if (whole) {
        xv[D][r] = load8<float, AL>(x[r] + k);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) xv[D][r].set(e, e < n ? x[r][k + e] : 0.f);
      }
    }
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      if (KCC && whole) {
        wv8[D][c] = load8<float, AL>(w[c] + k);
      } else if (whole) {
#pragma unroll
        for (int e = 0; e < 8; ++e) wv8[D][c].set(e, w[c][(k + e) * co.ld]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) wv8[D][c].set(e, e < n ? w[c][KCC ? k + e : (k + e) * co.ld] : 0.f);
      }
    }
  };
  f4 acc[CT][RT];
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int r = 0; r < RT; ++r) acc[c][r] = f4{0.f, 0.f, 0.f, 0.f};
  auto multiply = [&](auto d_) {
    constexpr int D = decltype(d_)::value;
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int r = 0; r < RT; ++r)
          acc[c][r] = __builtin_amdgcn_mfma_f32_16x16x4f32(wv8[D][c].get(e), xv[D][r].get(e), acc[c][r], 0, 0, 0);
  };
  int k = wv < 4 ? 32 * wv : K;   // (a larger block's other waves only keep the barrier)
  if (k < K) load(Int<0>{}, k);
  for (; k < K; k += 256) {
    if (k + 128 < K) load(Int<1>{}, k + 128);
    multiply(Int<0>{});
    if (k + 256 < K) load(Int<0>{}, k + 256);
    if (k + 128 < K) multiply(Int<1>{});
  }
  f4* part = reinterpret_cast<f4*>(lds);   // [tile][wave][lane]
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int r = 0; r < RT; ++r)
      if (wv < 4) part[((c * RT + r) * 4 + wv) * 64 + l] = acc[c][r];
  __syncthreads();
  if (wv < RT * CT) {   // a wave per tile
    const f4* t = part + wv * 256 + l;
    const f4 v = (t[0] + t[64]) + (t[128] + t[192]);
    const int m = 16 * (wv % RT) + i, n = 16 * (wv / RT) + 4 * g;
    if (m < ro.rows && n < co.rows) f(m, n, v, AL ? 4 : min(4, co.rows - n));
  }
}

// y = act(x W_g + b_g) + r: a tile of one group's rows per block, the epilogue on the
// sums in registers, so that z and y go out and r comes in once. 36864 x 2048 x 2048
// bfloat16 in eight groups, with z and r: 411 us; the products alone would take 300 at
// the card's 1.03 PFLOP/s for a plain product of that size, and the 600 MB of x, z, r
// and y 115 at a copy's rate, which only other blocks' products can hide.
template <class T, bool AL, class S>
__global__ void __launch_bounds__(S::NT) linear_fwd_kernel(LinearArgs<T> a) {
  __shared__ __align__(16) unsigned short lds[tile_lds<T, S>];
  const int tid = threadIdx.x;
  const int tiles_n = (a.n_out + S::BN - 1) / S::BN;
  const int id = xcd_order(block_id(), block_count());
  const int c0 = id % tiles_n * S::BN, cols = min(S::BN, a.n_out - c0);
  RowRun run;
  if (!find_run(a.offsets, a.groups, a.n, S::BM, id / tiles_n, run)) return;
  T* y = a.y + run.row0 * a.ldy + c0;
  T* z = a.z ? a.z + run.row0 * a.ldz + c0 : nullptr;
  if (run.group >= a.groups) {
    zero_rows(y, a.ldy, run.rows, cols, tid, S::NT);
    if (z) zero_rows(z, a.ldz, run.rows, cols, tid, S::NT);
    return;
  }
  f4 acc[S::TN][S::TM];
  const T* x = a.x + run.row0 * a.ldx;
  const T* w = a.w + (int64_t)run.group * a.n_in * a.n_out + c0;
  product<T, S, true, false, AL>({x, a.ldx, run.rows, 0, a.x + (a.n - 1) * a.ldx + a.n_in},
                                 {w, a.n_out, a.n_out - c0, 0, a.w + (int64_t)a.groups * a.n_in * a.n_out}, a.n_in, lds,
                                 tid, acc);
  linear_epilogue<T, AL, S>(a, run, c0, cols, y, z, tid, [&](int j, int i, auto b) { return lane_values<lane_width<T>>(acc, j, i) + b; });
}

template <bool AL, class S>
__global__ void __launch_bounds__(S::NT) linear_fwd_thin_kernel(LinearArgs<float> a) {
  __shared__ __align__(16) float lds[S::RT * S::CT * 1024];
  const int tid = threadIdx.x;
  const int tiles_n = (a.n_out + S::BN - 1) / S::BN;
  const int id = block_id();
  const int c0 = id % tiles_n * S::BN, cols = min(S::BN, a.n_out - c0);
  RowRun run;
  if (!find_run(a.offsets, a.groups, a.n, S::BM, id / tiles_n, run)) return;
  float* y = a.y + run.row0 * a.ldy + c0;
  float* z = a.z ? a.z + run.row0 * a.ldz + c0 : nullptr;
  if (run.group >= a.groups) {
    zero_rows(y, a.ldy, run.rows, cols, tid, S::NT);
    if (z) zero_rows(z, a.ldz, run.rows, cols, tid, S::NT);
    return;
  }
  const float* bias = a.bias ? a.bias + (int64_t)run.group * a.n_out + c0 : nullptr;
  const float* res = a.residual ? a.residual + run.row0 * a.ldr + c0 : nullptr;
  thin_product<S, false, AL>({a.x + run.row0 * a.ldx, a.ldx, run.rows, 0},
                             {a.w + (int64_t)run.group * a.n_in * a.n_out + c0, a.n_out, cols, 0}, a.n_in, lds, tid,
                             [&](int64_t m, int n, f4 v, int k) {
    if (bias) v += read_n<4>(bias + n, k, AL);
    if (z) store_n(z + m * a.ldz + n, v, k, AL);
#pragma unroll
    for (int q = 0; q < 4; ++q)
      v[q] = a.act == MACE_ACT_SILU ? activate<MACE_ACT_SILU>(v[q])
                                    : (a.act == MACE_ACT_GELU ? activate<MACE_ACT_GELU>(v[q]) : v[q]);
    if (res) v += read_n<4>(res + m * a.ldr + n, k, AL);
    store_n(y + m * a.ldy + n, v, k, AL);
  });
}

// Short sums (K up to 64 in FP32, 128 in 16 bits) over many rows: a wave keeps the
// weights of 64 columns in registers, as MFMA operands, and the run's rows go past
// them in chunks through LDS, where their parts lie split once for the block's four
// waves. The next chunk's rows are requested before this chunk's results are
// stored (memory operations complete in order: a later request would wait for
// the stores). Bound by the results' way to memory, against which the products (73 us
// at the matrix pipes' rate, FP32) are not wholly hidden: 81920 x 64 -> 1280 FP32 123
// to 145 us from card to card (as tiles 172 where it takes 144), 524288 x 64 -> 64
// bfloat16 38 us (3.5 TB/s; as tiles 53).
// KCC: the weights' rows are the columns of the result (dx).
template <class T, int KS_> struct NarrowShape {   // K <= 32 KS
  static constexpr int KS = KS_, BN = 256, NT = 256;
  static constexpr int CHUNK = sizeof(T) == 4 ? 64 : 128, RUN = sizeof(T) == 4 ? 256 : 512;   // rows per chunk, per block
  static constexpr int LDS = CHUNK * 32 * KS * Planes<T>::n;
};
template <class T, class S, bool KCC, bool AL, class F>
__device__ __forceinline__ void narrow_rows(const Operand<T>& ro, const T* w, int64_t ldw, int cols, int K,
                                            unsigned short* lds, int tid, F f) {
  constexpr int P = Planes<T>::n, KS = S::KS, C = 4 * KS, NV = S::CHUNK * C / S::NT, W = lane_width<T>;
  constexpr int PLANE = S::CHUNK * 32 * KS;
  const int l = tid & 63, wv = tid >> 6, i = l & 15, g = l >> 4, c0 = 64 * wv;
  // chunk rows of 4 KS vectors, XORed with the row (with the row pair at four vectors a row)
  auto place = [](int r, int c) { return (r * C + (c ^ (C == 4 ? r >> 1 & 3 : r & 7))) << 3; };
  Vec8<T> x[NV];
  auto load = [&](int m0) {
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int e = tid + S::NT * u, k = 8 * (e % C), n = K - k;   // n: k in bounds
      const T* p = ro.p + min(m0 + e / C, ro.rows - 1) * ro.ld + k;
      if constexpr (AL) {
        x[u].zero();
        if (n > 0) x[u] = load8<T, true>(p);
      } else {
        x[u] = load8_to<T, false>(p, ro.end);
        if (n < 8)
#pragma unroll
          for (int q = 0; q < 8; ++q)
            if (q >= n) x[u].set(q, (T)0.f);
      }
    }
  };
  load(0);
  us8 wr[4][KS][P];
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int64_t n = min(c0 + 16 * j + i, cols - 1);
      const int k = 32 * s + 8 * g;
      Vec8<T> v;
#pragma unroll
      for (int e = 0; e < 8; ++e) v.set(e, k + e < K ? w[KCC ? n * ldw + k + e : (k + e) * ldw + n] : (T)0.f);
      to_planes<T>(v, wr[j][s]);
    }
  for (int m0 = 0; m0 < ro.rows; m0 += S::CHUNK) {
    if (m0) __syncthreads();   // the previous chunk has been read
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int e = tid + S::NT * u;
      us8 q[P];
      to_planes<T>(x[u], q);
#pragma unroll
      for (int p = 0; p < P; ++p) *reinterpret_cast<us8*>(lds + p * PLANE + place(e / C, e % C)) = q[p];
    }
    __syncthreads();
    if (m0 + S::CHUNK < ro.rows) load(m0 + S::CHUNK);
    const int top = min(S::CHUNK, ro.rows - m0);
    for (int m = 0; m < top; m += 16) {
      f4 acc[4][1];
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j][0] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        us8 xb[1][P];
#pragma unroll
        for (int p = 0; p < P; ++p)
          xb[0][p] = *reinterpret_cast<const us8*>(lds + p * PLANE + place(m + i, 4 * s + g));
#pragma unroll
        for (int j = 0; j < 4; ++j) products<T>(wr[j][s], xb, acc[j]);
      }
#pragma unroll
      for (int j = 0; j < lane_vectors<4, W>; ++j) {
        const auto v = lane_values<W>(acc, j, 0);
        const int n = c0 + lane_column<W>(j, l);
        if (m + i < top && n < cols) f((int64_t)(m0 + m + i), n, v, AL ? W : min(W, cols - n));
      }
    }
  }
}

template <class T, bool AL, class S>
__global__ void __launch_bounds__(S::NT) __attribute__((amdgpu_waves_per_eu(2))) linear_fwd_narrow_kernel(LinearArgs<T> a) {
  __shared__ __align__(16) unsigned short lds[S::LDS];
  const int tid = threadIdx.x;
  const int tiles_n = (a.n_out + S::BN - 1) / S::BN;
  const int id = xcd_order(block_id(), block_count());
  const int c0 = id % tiles_n * S::BN, cols = min(S::BN, a.n_out - c0);
  RowRun run;
  if (!find_run(a.offsets, a.groups, a.n, S::RUN, id / tiles_n, run)) return;
  T* y = a.y + run.row0 * a.ldy + c0;
  T* z = a.z ? a.z + run.row0 * a.ldz + c0 : nullptr;
  if (run.group >= a.groups) {
    zero_rows(y, a.ldy, run.rows, cols, tid, S::NT);
    if (z) zero_rows(z, a.ldz, run.rows, cols, tid, S::NT);
    return;
  }
  const T* bias = a.bias ? a.bias + (int64_t)run.group * a.n_out + c0 : nullptr;
  const T* res = a.residual ? a.residual + run.row0 * a.ldr + c0 : nullptr;
  auto finish = [&](auto act) {
    narrow_rows<T, S, false, AL>({a.x + run.row0 * a.ldx, a.ldx, run.rows, 0, a.x + (a.n - 1) * a.ldx + a.n_in},
                                 a.w + (int64_t)run.group * a.n_in * a.n_out + c0, a.n_out, cols, a.n_in, lds, tid,
                                 [&](int64_t m, int n, auto v, int k) {
      constexpr int W = width_of<decltype(v)>;
      decltype(v) r = {};
      if (res) r = read_n<W>(res + m * a.ldr + n, k, AL);
      if (bias) v += read_n<W>(bias + n, k, AL);
      if (z) store_n(z + m * a.ldz + n, v, k, AL);
#pragma unroll
      for (int q = 0; q < W; ++q) v[q] = activate<decltype(act)::value>(v[q]);
      if (res) v += r;
      store_n(y + m * a.ldy + n, v, k, AL);
    });
  };
  if (a.act == MACE_ACT_SILU) finish(Int<MACE_ACT_SILU>{});
  else if (a.act == MACE_ACT_GELU) finish(Int<MACE_ACT_GELU>{});
  else finish(Int<MACE_ACT_NONE>{});
}

template <class T, bool AL, class S>
__global__ void __launch_bounds__(S::NT) __attribute__((amdgpu_waves_per_eu(2))) linear_row_grad_narrow_kernel(RowGradArgs<T> a) {
  __shared__ __align__(16) unsigned short lds[S::LDS];
  const int tid = threadIdx.x;
  const int tiles_n = (a.n_in + S::BN - 1) / S::BN;
  const int id = xcd_order(block_id(), block_count());
  const int c0 = id % tiles_n * S::BN, cols = min(S::BN, a.n_in - c0);
  RowRun run;
  if (!find_run(a.offsets, a.groups, a.n, S::RUN, id / tiles_n, run)) return;
  T* dx = a.dx + run.row0 * a.lddx + c0;
  if (run.group >= a.groups) {
    zero_rows(dx, a.lddx, run.rows, cols, tid, S::NT);
    return;
  }
  narrow_rows<T, S, true, AL>({a.dz + run.row0 * a.lddz, a.lddz, run.rows, 0, a.dz + (a.n - 1) * a.lddz + a.n_out},
                              a.w + ((int64_t)run.group * a.n_in + c0) * a.n_out, a.n_out, cols, a.n_out, lds, tid,
                              [&](int64_t m, int n, auto v, int k) {
    store_n(dx + m * a.lddx + n, without_factor(a, run.row0 + m, v), k, AL);
  });
}

// dx = dz W_g^T: tile `id`
template <class T, bool AL, class S>
__device__ __forceinline__ void row_grad_tile(const RowGradArgs<T>& a, int id, unsigned short* lds, int tid) {
  const int tiles_n = (a.n_in + S::BN - 1) / S::BN;
  const int c0 = id % tiles_n * S::BN, cols = min(S::BN, a.n_in - c0);
  RowRun run;
  if (!find_run(a.offsets, a.groups, a.n, S::BM, id / tiles_n, run)) return;
  T* dx = a.dx + run.row0 * a.lddx + c0;
  if (run.group >= a.groups) {
    zero_rows(dx, a.lddx, run.rows, cols, tid, S::NT);
    return;
  }
  f4 acc[S::TN][S::TM];
  const T* dz = a.dz + run.row0 * a.lddz;
  const T* w = a.w + ((int64_t)run.group * a.n_in + c0) * a.n_out;
  product<T, S, true, true, AL>({dz, a.lddz, run.rows, 0, a.dz + (a.n - 1) * a.lddz + a.n_out},
                                {w, a.n_out, cols, 0, a.w + (int64_t)a.groups * a.n_in * a.n_out}, a.n_out, lds, tid, acc);
  for_results<S, lane_width<T>, AL>(acc, run.rows, cols, tid, [&](int m, int n, auto v, int k) {
    store_n(dx + m * a.lddx + n, without_factor(a, run.row0 + m, v), k, AL);
  });
}

template <bool AL, class S>
__device__ __forceinline__ void row_grad_thin(const RowGradArgs<float>& a, int id, float* lds, int tid) {
  const int tiles_n = (a.n_in + S::BN - 1) / S::BN;
  const int c0 = id % tiles_n * S::BN, cols = min(S::BN, a.n_in - c0);
  RowRun run;
  if (!find_run(a.offsets, a.groups, a.n, S::BM, id / tiles_n, run)) return;
  float* dx = a.dx + run.row0 * a.lddx + c0;
  if (run.group >= a.groups) {
    zero_rows(dx, a.lddx, run.rows, cols, tid, S::NT);
    return;
  }
  thin_product<S, true, AL>({a.dz + run.row0 * a.lddz, a.lddz, run.rows, 0},
                            {a.w + ((int64_t)run.group * a.n_in + c0) * a.n_out, a.n_out, cols, 0}, a.n_out, lds, tid,
                            [&](int64_t m, int n, f4 v, int k) { store_n(dx + m * a.lddx + n, v, k, AL); });
}

// dW_g = x_g^T dz_g, the group's rows cut into `splits` parts: tile `id`
template <class T, bool AL, class S>
__device__ __forceinline__ void weight_grad_tile(const WeightGradArgs<T>& a, int id, unsigned short* lds, int tid) {
  const int tiles_n = (a.n_out + S::BN - 1) / S::BN, tiles_m = (a.n_in + S::BM - 1) / S::BM;
  const int c0 = id % tiles_n * S::BN;
  id /= tiles_n;
  const int m0 = id % tiles_m * S::BM;
  id /= tiles_m;
  const int split = id % a.splits, g = id / a.splits;
  const int rows = min(S::BM, a.n_in - m0), cols = min(S::BN, a.n_out - c0);
  int64_t r0 = 0, r1 = a.n;
  if (a.offsets) {
    r0 = min<int64_t>(max(a.offsets[g], 0), a.n);
    r1 = max<int64_t>(r0, min<int64_t>(max(a.offsets[g + 1], 0), a.n));
  }
  const int64_t per = ((r1 - r0 + a.splits - 1) / a.splits + S::BK - 1) / S::BK * S::BK;
  const int64_t k0 = min(r1, r0 + split * per), k1 = min(r1, k0 + per);
  f4 acc[S::TN][S::TM];
  product<T, S, false, false, AL>({a.x + k0 * a.ldx + m0, a.ldx, a.n_in - m0, 0, a.x + (a.n - 1) * a.ldx + a.n_in},
                                  {a.dz + k0 * a.lddz + c0, a.lddz, a.n_out - c0, 0, a.dz + (a.n - 1) * a.lddz + a.n_out},
                                  (int)(k1 - k0), lds, tid, acc);
  const int64_t at = ((int64_t)g * a.n_in + m0) * a.n_out + c0;
  if (a.part) {
    float* o = a.part + (int64_t)split * a.groups * a.n_in * a.n_out + at;
    for_results<S, 4, AL>(acc, rows, cols, tid,
                          [&](int m, int n, f4 v, int k) { store_n(o + (int64_t)m * a.n_out + n, v, k, AL); });
  } else {
    T* o = a.dw + at;
    for_results<S, lane_width<T>, AL>(acc, rows, cols, tid,
                                      [&](int m, int n, auto v, int k) { store_n(o + (int64_t)m * a.n_out + n, v, k, AL); });
  }
}

// db_g: the column sums of the group's runs (sums, one row per run), four row
// lanes, then in order: 64 columns of one group
template <class T>
__device__ __forceinline__ void bias_grad(const BiasGradArgs<T>& a, int id, float* lds, int tid) {
  const int blocks = (a.n_out + 63) / 64, g = id / blocks;
  if (g >= a.groups) return;   // (a grid's last row is full)
  const int c = tid & 63, y = tid >> 6, col = id % blocks * 64 + c;   // (waves past the fourth only keep the barrier)
  int first = 0, runs = 0;
  if (!a.offsets) {
    runs = (int)((a.n + a.run_rows - 1) / a.run_rows);
  } else {   // every wave sums the runs of the groups before g
    for (int e0 = 0; e0 <= g; e0 += 64) {
      const int e = e0 + c;
      int64_t p = 0, q = 0;
      if (e <= g) {
        p = min<int64_t>(max(a.offsets[e], 0), a.n);
        q = min<int64_t>(max(a.offsets[e + 1], 0), a.n);
      }
      const int r = q > p ? (int)((q - p + a.run_rows - 1) / a.run_rows) : 0;
      int before = e < g ? r : 0;
#pragma unroll
      for (int d = 32; d; d >>= 1) before += __shfl_xor(before, d);
      first += before;
      if (g - e0 < 64) runs = __shfl(r, g - e0);
    }
  }
  runs = min(runs, a.max_runs - first);   // (offsets that do not rise could count more runs than there are sums)
  float s = 0.f;
  if (col < a.n_out && y < 4)
    for (int r = y; r < runs; r += 32) {   // eight loads in flight, added in order
      float v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = a.sums[(int64_t)(first + min(r + 4 * u, runs - 1)) * a.n_out + col];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (r + 4 * u < runs) s += v[u];
    }
  if (y < 4) lds[y * 64 + c] = s;
  __syncthreads();
  if (y == 0 && col < a.n_out) a.db[(int64_t)g * a.n_out + col] = (T)(s + lds[64 + c] + lds[128 + c] + lds[192 + c]);
}

// All three gradients in one launch: blocks below row_blocks form dx, the next
// weight_blocks dW, the rest db. A small layer's step is bound by its launches;
// 36864 x 2048 x 2048 bfloat16 in eight groups 638 us, 0.97 PFLOP/s, bound by the
// products.
// RS: the shape of dx's tiles, S or a thin one.
template <class T, bool AL, class S, class RS>
__global__ void __launch_bounds__(S::NT)
linear_grad_kernel(RowGradArgs<T> a, WeightGradArgs<T> b, BiasGradArgs<T> c, int row_blocks, int weight_blocks) {
  __shared__ __align__(16) unsigned short lds[tile_lds<T, S>];
  const int tid = threadIdx.x;
  int id = block_id();
  if (id < row_blocks) {
    if constexpr (__is_same(S, RS)) row_grad_tile<T, AL, S>(a, xcd_order(id, row_blocks), lds, tid);
    else row_grad_thin<AL, RS>(a, id, reinterpret_cast<float*>(lds), tid);
  } else if ((id -= row_blocks) < weight_blocks) {
    weight_grad_tile<T, AL, S>(b, xcd_order(id, weight_blocks), lds, tid);
  } else {
    bias_grad<T>(c, id - weight_blocks, reinterpret_cast<float*>(lds), tid);
  }
}

// sum of the splits, in their order
template <class T>
__global__ void __launch_bounds__(256) linear_join_kernel(const float* __restrict__ part, int splits, int64_t size,
                                                          T* __restrict__ out) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= size) return;
  const bool vec = size % 4 == 0;   // (part and out begin at multiples of 16 bytes, or vec is not taken)
  const int k = (int)min<int64_t>(4, size - i);
  f4 s = {0.f, 0.f, 0.f, 0.f};
  for (int p = 0; p < splits; p += 8) {   // eight loads in flight, added in order
    f4 v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = read_n<4>(part + min(p + u, splits - 1) * size + i, k, vec);
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (p + u < splits) s += v[u];
  }
  const bool out_vec = vec && (reinterpret_cast<uintptr_t>(out) & (4 * sizeof(T) - 1)) == 0;
  store_n(out + i, s, k, out_vec);
}

// eight z of a row
template <class Z, bool AL>
struct SlopeValues {
  Vec8<Z> v;
  __device__ __forceinline__ void load(const Z* p, const Z* end, const float*, int64_t) { v = load8_to<Z, AL>(p, end); }
  __device__ __forceinline__ float get(int i) const { return v.get(i); }
};
template <bool AL>
struct SlopeValues<int8_t, AL> {   // (8-bit rows are padded to whole vectors)
  uint2 q;
  float s;
  __device__ __forceinline__ void load(const int8_t* p, const int8_t*, const float* zs, int64_t row) {
    q = *reinterpret_cast<const uint2*>(p);
    s = zs[row];
  }
  __device__ __forceinline__ float get(int i) const { return s * (float)(int8_t)((i < 4 ? q.x : q.y) >> 8 * (i & 3)); }
};

// dz = dy act'(z) over a run of rows (where there is an activation), and the
// run's column sums. A block takes 8 CX columns; its kSlopeThreads / CX row lanes
// each sum their rows, then are added in order. One pass over dy and z (36864 x 2048
// bfloat16: 101 to 115 us from card to card, 4.5 to 3.9 TB/s); both products read the rounded dz, so that the
// activation is not evaluated again for every tile of columns.
// Z: T, or int8_t with a scale for each row (z stands as q s, in FP32). xs: scales of an 8-bit input,
// or NULL; their split_scale8 factors go onto dz's rows before it is rounded, and the input's
// operand is exact: one rounding of the weights' gradients' terms, not two (error of
// bfloat16 gradients 2.3e-3, with x rounded instead 2.9e-3, of binary16 ones 2.9e-4 and 3.5e-4).
// That operand is written by the launch's further columns of blocks (Input8).
constexpr int kSlopeThreads = 1024;
template <class T>
struct Input8 {
  const int8_t* values;
  int64_t ld_values;
  T* x;         // its integers times the power of their scale, in FP32 times the scale; or NULL
  int64_t ld;   // a multiple of 8
  int n_in, cx;
  unsigned first;   // column of blocks
};
template <class T>
__device__ __forceinline__ void write_input8(const Input8<T>& in, const float* __restrict__ xs, const RowRun& run) {
  const int c = threadIdx.x % in.cx, col = 8 * ((blockIdx.y - in.first) * in.cx + c);
  if (col >= in.n_in) return;
  for (int r = threadIdx.x / in.cx; r < run.rows; r += kSlopeThreads / in.cx) {
    const int64_t row = run.row0 + r;
    const uint2 q = *reinterpret_cast<const uint2*>(in.values + row * in.ld_values + col);
    float s = xs[row], factor;
    if constexpr (sizeof(T) == 2) split_scale8<T>(s, s, factor);
    Vec8<T> v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v.set(i, (T)(s * (float)(int8_t)((i < 4 ? q.x : q.y) >> 8 * (i & 3))));
    *reinterpret_cast<Vec8<T>*>(in.x + row * in.ld + col) = v;
  }
}
template <class T, bool AL, class Z>
__global__ void __launch_bounds__(kSlopeThreads)
linear_slope_kernel(const T* __restrict__ dy, int64_t lddy, const Z* __restrict__ z, int64_t ldz,
                    const float* __restrict__ zs, const float* __restrict__ xs, T* __restrict__ dz,
                    int64_t lddz, float* __restrict__ sums, const int* __restrict__ offsets, int groups, int64_t n,
                    int n_out, int act, int run_rows, int cx, Input8<T> in) {
  __shared__ float red[kSlopeThreads * 8];
  RowRun run;
  if (!find_run(offsets, groups, n, run_rows, blockIdx.x, run) || run.group >= groups) return;
  if constexpr (__is_same(Z, int8_t))
    if (blockIdx.y >= in.first) return write_input8(in, xs, run);
  const int tid = threadIdx.x, c = tid % cx, ry = tid / cx, R = kSlopeThreads / cx;
  const int col = 8 * (blockIdx.y * cx + c), k = n_out - col;
  float s[8] = {};
  const T* dy_end = dy + (n - 1) * lddy + n_out;
  const Z* z_end = z ? z + (n - 1) * ldz + n_out : nullptr;
  constexpr int U = 2;   // rows in flight
  if (k > 0)
    for (int r0 = ry; r0 < run.rows; r0 += U * R) {
      Vec8<T> g[U];
      SlopeValues<Z, AL> v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t row = run.row0 + min(r0 + u * R, run.rows - 1);
        g[u] = load8_to<T, AL>(dy + row * lddy + col, dy_end);
        if (dz) v[u].load(z + row * ldz + col, z_end, zs, row);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (r0 + u * R >= run.rows) continue;
        if (dz) {
          float power, factor = 1.f;
          if constexpr (sizeof(T) == 2 && __is_same(Z, int8_t))
            if (xs) split_scale8<T>(xs[run.row0 + r0 + u * R], power, factor);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float o = g[u].get(i) * activation_slope(v[u].get(i), act);
            s[i] += o;
            g[u].set(i, (T)(factor * o));
          }
          *reinterpret_cast<Vec8<T>*>(dz + (run.row0 + r0 + u * R) * lddz + col) = g[u];   // (own buffer: rows padded to whole vectors)
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) s[i] += g[u].get(i);
        }
      }
    }
  if (!sums) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) red[(ry * cx + c) * 8 + i] = s[i];
  __syncthreads();
  for (int i = tid; i < 8 * cx; i += kSlopeThreads) {
    float t = 0.f;
    for (int r = 0; r < R; ++r) t += red[r * cx * 8 + i];
    const int o = 8 * blockIdx.y * cx + i;
    if (o < n_out) sums[(int64_t)blockIdx.x * n_out + o] = t;
  }
}

// ------------------------------------------------------------------ host
constexpr int kMaxLinearGroups = 1024;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool near(int64_t ld) { return ld <= 1 << 20; }   // a tile's rows lie within 32-bit byte offsets
size_t size_of(int dtype) { return dtype == MACE_TYPE_FP32 ? 4 : 2; }
size_t round256(size_t b) { return (b + 255) & ~size_t(255); }

mace_status check(const mace_linear_desc* d) {
  if (!d || d->n_rows < 0 || d->n_in < 1 || d->n_out < 1 || d->n_groups < 1) return MACE_EINVAL;
  if (d->dtype < MACE_TYPE_FP32 || d->dtype > MACE_TYPE_FP16 || d->act < MACE_ACT_NONE || d->act > MACE_ACT_GELU)
    return MACE_EINVAL;
  if (d->ld_x < d->n_in || d->ld_y < d->n_out || d->ld_residual < d->n_out || d->ld_preact < d->n_out) return MACE_EINVAL;
  if (d->n_rows > (1 << 30) || d->n_in > (1 << 20) || d->n_out > (1 << 20) || d->n_groups > kMaxLinearGroups)
    return MACE_EUNSUPPORTED;
  return MACE_OK;
}

// rows per run of the column sums: at most about 512 runs, so that joining them stays short
int slope_run(int64_t n) { return (int)(std::max<int64_t>(1, ceil_div(n, 64 * 512)) * 64); }
int64_t slope_runs(const mace_linear_desc& d) { return ceil_div(d.n_rows, slope_run(d.n_rows)) + d.n_groups; }

// Which tile a launch takes, by the blocks it would give 256 CUs. Large from
// kLargeBlocks of its own on: 8192 x 2048 x 2048 bfloat16 (256 of them) 71 us against
// 79 as Mid, 8192 x 1024 x 1024 (128) 34 against 24. Mid from kFillBlocks on:
// 8192 x 512 x 512 (256) bfloat16 10.3 us against 12.1 as Small, FP32 34 against 39;
// 4096 x 512 x 512 (128) 9.0 against 7.7, FP32 30 against 20.
constexpr int64_t kFillBlocks = 256, kLargeBlocks = 192;

// 256 x 256 keeps the matrix pipes busiest (two waves per SIMD, 128 x 64 results
// each); the others trade that for more blocks. FP32 is split as it is staged, so
// its tiles hold three planes per operand; with eight waves a block's splitting
// overlaps its products (4096 x 1024 x 1024: 57 us, four waves 67; 4730 x 1978 -> 178:
// 53 us, four waves 70). Where several such blocks share a CU they overlap each other, and
// four waves take 36864 x 2048 x 2048 in 1529 us against 1546, 36864 x 1023 x 1023 in 425
// against 458, but their dx in 1500 against 1462 and 410 against 405. 16-bit operands at
// any alignment stay with eight (36864 x 1023 x 1023: 135 us, four waves 144).
template <class T, bool AL> struct Shapes {   // (16-bit, any alignment)
  using Mid = TileShape<128, 128, 4, 2, 64, 1>;
  using Large = Mid;
  using Small = TileShape<64, 64, 2, 2, 64, 2>;
};
template <> struct Shapes<__bf16, true> {
  using Large = TileShape<256, 256, 2, 4, 64, 2, true>;
  using Mid = TileShape<128, 128, 2, 2, 64, 2, true>;
  using Small = TileShape<64, 64, 2, 2, 64, 4, true>;
};
template <> struct Shapes<_Float16, true> : Shapes<__bf16, true> {};
template <> struct Shapes<float, false> {
  using Large = TileShape<128, 128, 2, 2, 32, 1>;
  using Mid = TileShape<128, 128, 4, 2, 32, 1>;
  using Small = TileShape<64, 64, 2, 4, 64, 1>;
};
template <> struct Shapes<float, true> : Shapes<float, false> {};
using Thin = ThinShape<1, 1>;
using Thin2 = ThinShape<2, 2>;
// FP32 launches of fewer than kThinBlocks 64 x 64 tiles; Thin2 from kFillBlocks of
// its own. 16 x 2048 x 2048 (32 tiles) 12 us against 36 as Small, 256 x 1024 x 1024
// (64) 11 against 20, 192 x 2048 x 2048 (96) 37 against 38, 320 x 256 x 1536 (120) 8.1
// against 7.6, 640 x 1024 x 1024 (160) 31 against 24.
constexpr int64_t kThinBlocks = 96;
bool thin(int64_t rows, int64_t cols) { return ceil_div(rows, 64) * ceil_div(cols, 64) < kThinBlocks; }
bool thin2(int64_t rows, int64_t cols) { return ceil_div(rows, 32) * ceil_div(cols, 32) >= kFillBlocks; }
// Sums of K short enough for narrow_rows, and rows for at least kNarrowBlocks waves of
// 64 columns and 512 rows: four per SIMD, so that their weights' loads are hidden.
// FP32 sums of more than 32 products also need more than kNarrowColumns columns, as a
// wave splits its rows for 64 columns at a time: 262144 x 64 -> 192 74 us against 94
// as tiles, -> 128 74 against 62, 524288 x 64 -> 64 105 against 80 (32 -> 64: 55
// against 61; bfloat16, 64 -> 64: 38 against 53).
constexpr int64_t kNarrowBlocks = 1024, kNarrowColumns = 128;
template <class T> bool narrow(int64_t rows, int64_t cols, int K) {
  if (sizeof(T) == 4 && K > 32 && cols <= kNarrowColumns) return false;
  return K <= (sizeof(T) == 4 ? 64 : 128) && ceil_div(rows, 512) * ceil_div(cols, 64) >= kNarrowBlocks;
}
template <class T, class F>
mace_status with_narrow(int K, F f) {
  if (K <= 32) return f(NarrowShape<T, 1>{});
  if constexpr (sizeof(T) == 2)
    if (K > 64) return f(NarrowShape<T, 4>{});
  return f(NarrowShape<T, 2>{});
}
enum { kSmall, kMid, kLarge };
// runs: the groups that the rows are cut at; where they are short, a 256-row tile
// would hold too few rows
int shape_of(int64_t rows, int64_t cols, int64_t batch = 1, int64_t runs = 1) {
  if ((runs == 1 || rows / runs >= 512) && ceil_div(rows, 256) * ceil_div(cols, 256) * batch >= kLargeBlocks) return kLarge;
  return ceil_div(rows, 128) * ceil_div(cols, 128) * batch >= kFillBlocks ? kMid : kSmall;
}
// f(shape) for the kind of tile; shapes that are the same type are instantiated once
template <class T, bool AL, class F>
mace_status with_shape(int kind, F f) {
  if (kind == kLarge) return f(typename Shapes<T, AL>::Large{});
  if (kind == kMid) return f(typename Shapes<T, AL>::Mid{});
  return f(typename Shapes<T, AL>::Small{});
}

struct BackwardPlan {
  int weight_kind;
  int splits;
  int64_t lddz;
  size_t dz, sums, part, total;   // byte offsets
};

// kind of tile of dW's blocks, and the parts each group's rows are cut into:
// enough blocks to fill the chip, at least 512 rows each (of a group of mean size). Only
// aligned 16-bit rows have 256-wide tiles (20000 x 512 x 2048 FP32 222 us with the 8 parts
// that fill it, 231 with 16)
int weight_shape(const mace_linear_desc& d, int& splits) {
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>(64, d.n_rows / d.n_groups / 512));
  const int kind = shape_of(d.n_in, d.n_out, d.n_groups * most);
  const bool wide = kind == kLarge && d.dtype != MACE_TYPE_FP32 && ((d.n_in | d.n_out) & 7) == 0;
  const int b = wide ? 256 : (kind == kSmall ? 64 : 128);
  const int64_t tiles = ceil_div(d.n_in, b) * ceil_div(d.n_out, b) * d.n_groups;
  splits = (int)std::max<int64_t>(1, std::min(most, (wide ? 256 : 512) / tiles));
  return kind;
}

BackwardPlan plan_backward(const mace_linear_desc& d, bool bias, bool weights) {
  BackwardPlan p{};
  p.weight_kind = weight_shape(d, p.splits);
  p.lddz = (d.n_out + 7) / 8 * 8;
  size_t o = 0;
  p.dz = o;
  if (d.act != MACE_ACT_NONE) o += round256(size_t(d.n_rows) * p.lddz * size_of(d.dtype));
  p.sums = o;
  if (bias) o += round256(size_t(slope_runs(d)) * d.n_out * 4);
  p.part = o;
  if (weights && p.splits > 1) o += round256(size_t(p.splits) * d.n_groups * d.n_in * d.n_out * 4);
  p.total = o;
  return p;
}

template <class T>
mace_status forward(const mace_linear_desc& d, const void* x, const void* w, const void* bias, const void* residual,
                    const int* offsets, void* y, void* z, hipStream_t s) {
  LinearArgs<T> a{(const T*)x, (const T*)w, (const T*)bias, (const T*)residual, (T*)y, (T*)z, offsets, d.n_rows,
                  d.ld_x, d.ld_y, d.ld_residual, d.ld_preact, d.n_in, d.n_out, d.n_groups, d.act};
  const bool al = aligned16(x) && aligned16(w) && aligned16(bias) && aligned16(residual) && aligned16(y) &&
                  aligned16(z) && ((d.n_in | d.n_out | d.ld_x | d.ld_y | d.ld_residual | d.ld_preact) & 7) == 0 &&
                  near(d.ld_x);
  auto go = [&](auto al_) -> mace_status {
    constexpr bool AL = decltype(al_)::value;
    if (narrow<T>(d.n_rows, d.n_out, d.n_in))
      return with_narrow<T>(d.n_in, [&](auto shape) -> mace_status {
        using S = decltype(shape);
        const int64_t blocks = (ceil_div(d.n_rows, S::RUN) + (offsets ? d.n_groups : 0)) * ceil_div(d.n_out, S::BN);
        if (!fits_grid(blocks)) return MACE_EUNSUPPORTED;
        linear_fwd_narrow_kernel<T, AL, S><<<grid_of(blocks), S::NT, 0, s>>>(a);
        return launched();
      });
    if constexpr (sizeof(T) == 4)
      if (thin(d.n_rows, d.n_out)) {
        auto run = [&](auto shape) {
          using S = decltype(shape);
          const int64_t blocks = (ceil_div(d.n_rows, S::BM) + (offsets ? d.n_groups : 0)) * ceil_div(d.n_out, S::BN);
          linear_fwd_thin_kernel<AL, S><<<grid_of(blocks), S::NT, 0, s>>>(a);
          return launched();
        };
        return thin2(d.n_rows, d.n_out) ? run(Thin2{}) : run(Thin{});
      }
    return with_shape<T, AL>(shape_of(d.n_rows, d.n_out, 1, d.n_groups), [&](auto shape) -> mace_status {
      using S = decltype(shape);
      const int64_t blocks = (ceil_div(d.n_rows, S::BM) + (offsets ? d.n_groups : 0)) * ceil_div(d.n_out, S::BN);
      if (!fits_grid(blocks)) return MACE_EUNSUPPORTED;
      linear_fwd_kernel<T, AL, S><<<grid_of(blocks), S::NT, 0, s>>>(a);
      return launched();
    });
  };
  return al ? go(Int<1>{}) : go(Int<0>{});
}

template <class T, class Z = T>
mace_status backward(const mace_linear_desc& d, const void* dy, int64_t lddy, const void* x, const float* xs, Input8<T> in,
                     const void* w, const void* z, const float* zs, const int* offsets, void* dx, int64_t lddx, void* dw, void* db, char* ws, hipStream_t s) {
  const BackwardPlan p = plan_backward(d, db != nullptr, dw != nullptr);
  const T* dz = (const T*)dy;
  int64_t lddz = lddy;
  if (d.act != MACE_ACT_NONE) {
    dz = reinterpret_cast<T*>(ws + p.dz);
    lddz = p.lddz;
  }
  float* sums = reinterpret_cast<float*>(ws + p.sums);
  mace_status st = MACE_OK;
  if (d.n_rows > 0 && (d.act != MACE_ACT_NONE || db)) {
    const int vecs = (d.n_out + 7) / 8;
    int cx = 1;
    while (cx < 64 && cx < vecs) cx *= 2;
    const bool al = aligned16(dy) && (__is_same(Z, int8_t) || aligned16(z)) && ((d.n_out | lddy | d.ld_preact) & 7) == 0;
    const int vecs_in = (d.n_in + 7) / 8;
    in.cx = 1;
    while (in.cx < 64 && in.cx < vecs_in) in.cx *= 2;
    in.first = (unsigned)ceil_div(vecs, cx);
    const dim3 grid((unsigned)slope_runs(d), in.first + (in.x ? (unsigned)ceil_div(vecs_in, in.cx) : 0));
    T* out = d.act != MACE_ACT_NONE ? const_cast<T*>(dz) : nullptr;
    auto go = [&](auto f) {
      f<<<grid, kSlopeThreads, 0, s>>>((const T*)dy, lddy, (const Z*)z, d.ld_preact, zs, xs, out, lddz, db ? sums : nullptr, offsets,
                             d.n_groups, d.n_rows, d.n_out, d.act, slope_run(d.n_rows), cx, in);
    };
    if (al) go(linear_slope_kernel<T, true, Z>);
    else go(linear_slope_kernel<T, false, Z>);
    if ((st = launched()) != MACE_OK) return st;
  }
  const bool al = aligned16(dz) && aligned16(w) && aligned16(dx) && aligned16(x) && aligned16(dw) && near(lddz) &&
                  near(d.ld_x) && ((d.n_in | d.n_out | lddz | lddx | (dw ? d.ld_x : 0)) & 7) == 0;
  const RowGradArgs<T> ra{dz, (const T*)w, (T*)dx, offsets, d.n_rows, lddz, lddx, d.n_in, d.n_out, d.n_groups, xs};
  const WeightGradArgs<T> wa{(const T*)x, dz, (T*)dw, p.splits > 1 ? reinterpret_cast<float*>(ws + p.part) : nullptr,
                             offsets, d.n_rows, d.ld_x, lddz, d.n_in, d.n_out, d.n_groups, p.splits};
  const BiasGradArgs<T> ba{sums, (T*)db, offsets, d.n_rows, d.n_out, db ? d.n_groups : 0, slope_run(d.n_rows), (int)slope_runs(d)};
  bool want_x = dx && d.n_rows > 0;
  if (want_x && narrow<T>(d.n_rows, d.n_in, d.n_out)) {
    auto run = [&](auto al_) {
      constexpr bool AL = decltype(al_)::value;
      return with_narrow<T>(d.n_out, [&](auto shape) -> mace_status {
        using S = decltype(shape);
        const int64_t blocks = (ceil_div(d.n_rows, S::RUN) + (offsets ? d.n_groups : 0)) * ceil_div(d.n_in, S::BN);
        if (!fits_grid(blocks)) return MACE_EUNSUPPORTED;
        linear_row_grad_narrow_kernel<T, AL, S><<<grid_of(blocks), S::NT, 0, s>>>(ra);
        return launched();
      });
    };
    if ((st = al ? run(Int<1>{}) : run(Int<0>{})) != MACE_OK) return st;
    want_x = false;
  }
  const bool thin_x = sizeof(T) == 4 && want_x && thin(d.n_rows, d.n_in);
  // one launch for all three where dx and dW take the same kind of tile (thin
  // tiles of dx go with small ones of dW)
  auto go = [&](auto al_, int kind, bool rows, bool weights, bool bias) {
    constexpr bool AL = decltype(al_)::value;
    return with_shape<T, AL>(kind, [&](auto shape) -> mace_status {
      using S = decltype(shape);
      auto run = [&](auto row_shape) -> mace_status {
        using RS = decltype(row_shape);
        const int64_t rb = rows ? (ceil_div(d.n_rows, RS::BM) + (offsets ? d.n_groups : 0)) * ceil_div(d.n_in, RS::BN) : 0;
        const int64_t wb = weights ? ceil_div(d.n_in, S::BM) * ceil_div(d.n_out, S::BN) * d.n_groups * p.splits : 0;
        const int64_t blocks = rb + wb + (bias ? ceil_div(d.n_out, 64) * d.n_groups : 0);
        if (!fits_grid(blocks)) return MACE_EUNSUPPORTED;
        if (blocks == 0) return MACE_OK;
        linear_grad_kernel<T, AL, S, RS><<<grid_of(blocks), S::NT, 0, s>>>(ra, wa, ba, (int)rb, (int)wb);
        return launched();
      };
      if constexpr (sizeof(T) == 4 && S::BM == 64)
        if (rows && thin_x) return thin2(d.n_rows, d.n_in) ? run(Thin2{}) : run(Thin{});
      return run(S{});
    });
  };
  auto grads = [&](int kind, bool rows, bool weights, bool bias) {
    return al ? go(Int<1>{}, kind, rows, weights, bias) : go(Int<0>{}, kind, rows, weights, bias);
  };
  const int kind_x = shape_of(d.n_rows, d.n_in, 1, d.n_groups);
  if (!want_x || !dw || kind_x == p.weight_kind) {
    st = grads(dw ? p.weight_kind : kind_x, want_x, dw != nullptr, db != nullptr);
  } else {
    if ((st = grads(kind_x, true, false, db != nullptr)) != MACE_OK) return st;
    st = grads(p.weight_kind, false, true, false);
  }
  if (st != MACE_OK) return st;
  if (dw && p.splits > 1) {
    const int64_t size = (int64_t)d.n_groups * d.n_in * d.n_out;
    linear_join_kernel<T><<<(unsigned)ceil_div(size, 1024), 256, 0, s>>>(wa.part, p.splits, size, (T*)dw);
    st = launched();
  }
  return st;
}

}  // namespace
}  // namespace mace

using namespace mace;

extern "C" mace_status mace_linear_forward(const mace_linear_desc* desc, const void* x, const void* weights,
                                           const void* bias, const void* residual, const int32_t* group_offsets,
                                           void* y, void* preact, void* stream) {
  const mace_status st = check(desc);
  if (st != MACE_OK) return st;
  const mace_linear_desc& d = *desc;
  if (!weights || (d.n_rows > 0 && (!x || !y)) || (d.n_groups > 1 && !group_offsets)) return MACE_EINVAL;
  if (d.n_rows == 0) return MACE_OK;
  hipStream_t s = (hipStream_t)stream;
  if (d.dtype == MACE_TYPE_FP32) return forward<float>(d, x, weights, bias, residual, group_offsets, y, preact, s);
  if (d.dtype == MACE_TYPE_BF16) return forward<__bf16>(d, x, weights, bias, residual, group_offsets, y, preact, s);
  return forward<_Float16>(d, x, weights, bias, residual, group_offsets, y, preact, s);
}

extern "C" size_t mace_linear_backward_workspace_bytes(const mace_linear_desc* desc, int32_t want_bias, int32_t want_weights) {
  if (check(desc) != MACE_OK) return 0;
  return plan_backward(*desc, want_bias != 0, want_weights != 0).total + 256;
}

extern "C" mace_status mace_linear_backward(const mace_linear_desc* desc, const void* dy, int64_t ld_dy, const void* x,
                                            const void* weights, const void* preact, const int32_t* group_offsets,
                                            void* dx, int64_t ld_dx, void* dweights, void* dbias, void* workspace,
                                            size_t workspace_bytes, void* stream) {
  const mace_status st = check(desc);
  if (st != MACE_OK) return st;
  const mace_linear_desc& d = *desc;
  if (!weights || (d.n_groups > 1 && !group_offsets) || ld_dy < d.n_out || (dx && ld_dx < d.n_in)) return MACE_EINVAL;
  if (d.n_rows > 0 && (!dy || (dweights && !x) || (d.act != MACE_ACT_NONE && !preact))) return MACE_EINVAL;
  const BackwardPlan p = plan_backward(d, dbias != nullptr, dweights != nullptr);
  if (p.total > 0 && !workspace) return MACE_EINVAL;
  if (p.total > 0 && workspace_bytes < p.total + 256) return MACE_ENOSPACE;
  char* ws = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(workspace) + 255) & ~uintptr_t(255));
  hipStream_t s = (hipStream_t)stream;
  if (d.dtype == MACE_TYPE_FP32)
    return backward<float>(d, dy, ld_dy, x, nullptr, {}, weights, preact, nullptr, group_offsets, dx, ld_dx, dweights, dbias, ws, s);
  if (d.dtype == MACE_TYPE_BF16)
    return backward<__bf16>(d, dy, ld_dy, x, nullptr, {}, weights, preact, nullptr, group_offsets, dx, ld_dx, dweights, dbias, ws, s);
  return backward<_Float16>(d, dy, ld_dy, x, nullptr, {}, weights, preact, nullptr, group_offsets, dx, ld_dx, dweights, dbias, ws, s);
}

// The input's 8-bit rows are written out in dtype first, as the products' operand: beside dz where there is an
// activation (Input8), by a launch of their own otherwise.
namespace {
int64_t ld_input8(const mace_linear_desc& d) { return (d.n_in + 7) / 8 * 8; }
size_t input8_bytes(const mace_linear_desc& d, bool weights) {
  return weights ? round256(size_t(d.n_rows) * ld_input8(d) * size_of(d.dtype)) : 0;
}
mace_status check8(const mace_linear_desc* d) {
  const mace_status st = check(d);
  if (st != MACE_OK) return st;
  if (d->ld_x % 16 || (d->act != MACE_ACT_NONE && d->ld_preact % 16)) return MACE_EINVAL;
  const bool wide = d->act != MACE_ACT_NONE && (d->n_out > kMaxColumns8 || d->ld_preact > kMaxPitch8);
  return wide || d->n_in > kMaxColumns8 || d->ld_x > kMaxPitch8 ? MACE_EUNSUPPORTED : MACE_OK;
}
}  // namespace

extern "C" size_t mace_linear_backward8_workspace_bytes(const mace_linear_desc* desc, int32_t want_bias, int32_t want_weights) {
  if (check8(desc) != MACE_OK) return 0;
  return input8_bytes(*desc, want_weights != 0) + plan_backward(*desc, want_bias != 0, want_weights != 0).total + 256;
}

extern "C" mace_status mace_linear_backward8(const mace_linear_desc* desc, const void* dy, int64_t ld_dy, const void* x8,
                                             const float* x_scales, const void* weights, const void* z8,
                                             const float* z_scales, const int32_t* group_offsets, void* dx, int64_t ld_dx,
                                             void* dweights, void* dbias, void* workspace, size_t workspace_bytes,
                                             void* stream) {
  mace_status st = check8(desc);
  if (st != MACE_OK) return st;
  mace_linear_desc d = *desc;
  if (!weights || (d.n_groups > 1 && !group_offsets) || ld_dy < d.n_out || (dx && ld_dx < d.n_in)) return MACE_EINVAL;
  if (d.n_rows > 0) {
    if (!dy || (dweights && (!x8 || !x_scales || !aligned16(x8)))) return MACE_EINVAL;
    if (d.act != MACE_ACT_NONE && (!z8 || !z_scales || !aligned16(z8))) return MACE_EINVAL;
  }
  const size_t need = mace_linear_backward8_workspace_bytes(desc, dbias != nullptr, dweights != nullptr);
  if (need > 256 && !workspace) return MACE_EINVAL;
  if (need > 256 && workspace_bytes < need) return MACE_ENOSPACE;
  char* ws = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(workspace) + 255) & ~uintptr_t(255));
  hipStream_t s = (hipStream_t)stream;
  void* x = dweights && d.n_rows > 0 ? ws : nullptr;
  ws += input8_bytes(d, dweights != nullptr);
  if (x && d.act == MACE_ACT_NONE) {
    const mace_rows8_desc r{d.n_rows, d.n_in, d.dtype, ld_input8(d), d.ld_x};
    if ((st = mace_unpack_rows(&r, x8, x_scales, x, stream)) != MACE_OK) return st;
  }
  const int64_t ld_x8 = d.ld_x;
  d.ld_x = ld_input8(d);
  return by_type(d.dtype, [&](auto zero) {
    using T = decltype(zero);
    if (d.act == MACE_ACT_NONE)
      return backward<T>(d, dy, ld_dy, x, nullptr, {}, weights, nullptr, nullptr, group_offsets, dx, ld_dx, dweights, dbias, ws, s);
    const Input8<T> in{(const int8_t*)x8, ld_x8, (T*)x, d.ld_x, d.n_in};
    return backward<T, int8_t>(d, dy, ld_dy, x, x_scales, in, weights, z8, z_scales, group_offsets, dx, ld_dx, dweights, dbias,
                               ws, s);
  });
}
