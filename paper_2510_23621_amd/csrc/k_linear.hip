// Grouped dense layer y = act(x W_g + b_g) + r and its backward pass:
// mace_linear_forward, mace_linear_backward.
#include <algorithm>
#include <cmath>

#include "../../include/mace.h"
#include "dense.h"

namespace mace {
namespace {

// ------------------------------------------------------------------ activations
__device__ __forceinline__ float activate(float z, int act) {
  if (act == MACE_ACT_SILU) return silu(z);
  if (act == MACE_ACT_GELU) return 0.5f * z * erfcf(-0.70710678118654752f * z);   // z Phi(z)
  return z;
}
// act'(z); beyond |z| = 88 the slopes are 0 and 1 to FP32, and z (1 - s) would
// be inf 0 at an infinite z
__device__ __forceinline__ float activation_slope(float z, int act) {
  z = z > 88.f ? 88.f : (z < -88.f ? -88.f : z);   // (keeps NaN)
  if (act == MACE_ACT_SILU) return silu_grad(z);
  return 0.5f * erfcf(-0.70710678118654752f * z) + 0.39894228040143268f * z * exp_neg(0.5f * z * z);
}

// ------------------------------------------------------------------ arguments
template <class T>
struct LinearArgs {
  const T *x, *w, *bias, *residual;
  T *y, *z;
  const int* offsets;
  int64_t n, ldx, ldy, ldr, ldz;
  int n_in, n_out, groups, act;
};
template <class T>
struct RowGradArgs {
  const T *dz, *w;
  T* dx;
  const int* offsets;
  int64_t n, lddz, lddx;
  int n_in, n_out, groups;
};
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
  int n_out, run_rows, max_runs;
};

// rows behind the last group: zeros
template <class T>
__device__ __forceinline__ void zero_rows(T* y, int64_t ld, int rows, int cols, int tid, int nt) {
  for (int i = tid; i < rows * cols; i += nt) y[(int64_t)(i / cols) * ld + i % cols] = (T)0.f;
}

template <class T, bool AL, class S>
__global__ void __launch_bounds__(S::NT) linear_fwd_kernel(LinearArgs<T> a) {
  __shared__ __align__(16) unsigned short lds[tile_lds<T, S>];
  const int tid = threadIdx.x;
  const int tiles_n = (a.n_out + S::BN - 1) / S::BN;
  const int id = xcd_order(blockIdx.x, gridDim.x);
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
  TileSource<T, S::BM, S::BK, true, AL, S::NT> xr;
  TileSource<T, S::BN, S::BK, false, AL, S::NT> wc;
  xr.init(a.x + run.row0 * a.ldx, a.ldx, run.rows, tid);
  wc.init(a.w + (int64_t)run.group * a.n_in * a.n_out + c0, a.n_out, a.n_out - c0, tid);
  f4 acc[S::TN][S::TM];
  tile_gemm<T, S, true, false, AL>(xr, wc, a.n_in, lds, tid, acc);
  const T* bias = a.bias ? a.bias + (int64_t)run.group * a.n_out + c0 : nullptr;
  const T* res = a.residual ? a.residual + run.row0 * a.ldr + c0 : nullptr;
  for_results<S>(acc, run.rows, cols, tid, [&](int m, int n, f4 v, int k) {
    const bool vec = AL && k == 4;
    if (bias) v += read4(bias + n, k, vec);
    if (z) store4(z + m * a.ldz + n, v, k, vec);
    if (a.act != MACE_ACT_NONE)
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = activate(v[i], a.act);
    if (res) v += read4(res + m * a.ldr + n, k, vec);
    store4(y + m * a.ldy + n, v, k, vec);
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
  TileSource<T, S::BM, S::BK, true, AL, S::NT> zr;
  TileSource<T, S::BN, S::BK, true, AL, S::NT> wc;
  zr.init(a.dz + run.row0 * a.lddz, a.lddz, run.rows, tid);
  wc.init(a.w + ((int64_t)run.group * a.n_in + c0) * a.n_out, a.n_out, cols, tid);
  f4 acc[S::TN][S::TM];
  tile_gemm<T, S, true, true, AL>(zr, wc, a.n_out, lds, tid, acc);
  for_results<S>(acc, run.rows, cols, tid,
                 [&](int m, int n, f4 v, int k) { store4(dx + m * a.lddx + n, v, k, AL && k == 4); });
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
  TileSource<T, S::BM, S::BK, false, AL, S::NT> xr;
  TileSource<T, S::BN, S::BK, false, AL, S::NT> zc;
  xr.init(a.x + k0 * a.ldx + m0, a.ldx, a.n_in - m0, tid);
  zc.init(a.dz + k0 * a.lddz + c0, a.lddz, a.n_out - c0, tid);
  f4 acc[S::TN][S::TM];
  tile_gemm<T, S, false, false, AL>(xr, zc, (int)(k1 - k0), lds, tid, acc);
  const int64_t at = ((int64_t)g * a.n_in + m0) * a.n_out + c0;
  if (a.part) {
    float* o = a.part + (int64_t)split * a.groups * a.n_in * a.n_out + at;
    for_results<S>(acc, rows, cols, tid,
                   [&](int m, int n, f4 v, int k) { store4(o + (int64_t)m * a.n_out + n, v, k, AL && k == 4); });
  } else {
    T* o = a.dw + at;
    for_results<S>(acc, rows, cols, tid,
                   [&](int m, int n, f4 v, int k) { store4(o + (int64_t)m * a.n_out + n, v, k, AL && k == 4); });
  }
}

// db_g: the column sums of the group's runs (sums, one row per run), four row
// lanes, then in order: 64 columns of one group
template <class T>
__device__ __forceinline__ void bias_grad(const BiasGradArgs<T>& a, int id, float* lds, int tid) {
  const int blocks = (a.n_out + 63) / 64, g = id / blocks;
  const int c = tid & 63, y = tid >> 6, col = id % blocks * 64 + c;
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
  if (col < a.n_out)
    for (int r = y; r < runs; r += 4) s += a.sums[(int64_t)(first + r) * a.n_out + col];
  lds[y * 64 + c] = s;
  __syncthreads();
  if (y == 0 && col < a.n_out) a.db[(int64_t)g * a.n_out + col] = (T)(s + lds[64 + c] + lds[128 + c] + lds[192 + c]);
}

// All three gradients in one launch: blocks below row_blocks form dx, the next
// weight_blocks dW, the rest db.
template <class T, bool ALX, bool ALW, class S>
__global__ void __launch_bounds__(S::NT)
linear_grad_kernel(RowGradArgs<T> a, WeightGradArgs<T> b, BiasGradArgs<T> c, int row_blocks, int weight_blocks) {
  __shared__ __align__(16) unsigned short lds[tile_lds<T, S>];
  const int tid = threadIdx.x;
  int id = blockIdx.x;
  if (id < row_blocks) {
    row_grad_tile<T, ALX, S>(a, xcd_order(id, row_blocks), lds, tid);
  } else if ((id -= row_blocks) < weight_blocks) {
    weight_grad_tile<T, ALW, S>(b, xcd_order(id, weight_blocks), lds, tid);
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
  f4 s = read4(part + i, k, vec);
  for (int p = 1; p < splits; ++p) s += read4(part + p * size + i, k, vec);
  const bool out_vec = vec && (reinterpret_cast<uintptr_t>(out) & (4 * sizeof(T) - 1)) == 0;
  store4(out + i, s, k, out_vec);
}

// dz = dy act'(z) over a run of rows (where there is an activation), and the
// run's column sums. A block takes 8 CX columns; its 256 / CX row lanes each sum
// their rows, then are added in order.
template <class T, bool AL>
__global__ void __launch_bounds__(256)
linear_slope_kernel(const T* __restrict__ dy, int64_t lddy, const T* __restrict__ z, int64_t ldz, T* __restrict__ dz,
                    int64_t lddz, float* __restrict__ sums, const int* __restrict__ offsets, int groups, int64_t n,
                    int n_out, int act, int run_rows, int cx) {
  __shared__ float red[256 * 8];
  RowRun run;
  if (!find_run(offsets, groups, n, run_rows, blockIdx.x, run) || run.group >= groups) return;
  const int tid = threadIdx.x, c = tid % cx, ry = tid / cx, R = 256 / cx;
  const int col = 8 * (blockIdx.y * cx + c), k = n_out - col;
  float s[8] = {};
  if (k > 0)
    for (int r = ry; r < run.rows; r += R) {
      const int64_t row = run.row0 + r;
      Vec8<T> g = load8_upto<T, AL>(dy + row * lddy + col, k);
      if (dz) {
        const Vec8<T> v = load8_upto<T, AL>(z + row * ldz + col, k);
        float o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = g.get(i) * activation_slope(v.get(i), act);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          s[i] += o[i];
          g.set(i, (T)o[i]);
        }
        if (k >= 8) *reinterpret_cast<Vec8<T>*>(dz + row * lddz + col) = g;   // (own buffer: aligned rows)
        else for (int i = 0; i < k; ++i) dz[row * lddz + col + i] = (T)o[i];
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] += g.get(i);
      }
    }
  if (!sums) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) red[(ry * cx + c) * 8 + i] = s[i];
  __syncthreads();
  for (int i = tid; i < 8 * cx; i += 256) {
    float t = 0.f;
    for (int r = 0; r < R; ++r) t += red[r * cx * 8 + i];
    const int o = 8 * blockIdx.y * cx + i;
    if (o < n_out) sums[(int64_t)blockIdx.x * n_out + o] = t;
  }
}

// ------------------------------------------------------------------ host
constexpr int kMaxLinearGroups = 1024;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
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

// parts each group's rows are cut into for dW: enough blocks to fill the chip, at least 512 rows each
int weight_splits(const mace_linear_desc& d, int bm, int bn) {
  const int64_t tiles = ceil_div(d.n_in, bm) * ceil_div(d.n_out, bn) * d.n_groups;
  const int64_t want = 512 / std::max<int64_t>(1, tiles), most = d.n_rows / d.n_groups / 512;
  return (int)std::max<int64_t>(1, std::min({want, most, (int64_t)64}));
}

constexpr int64_t kFillBlocks = 256;   // blocks from which the larger tile is taken (one per CU)

struct BackwardPlan {
  int splits;
  int64_t lddz;
  size_t dz, sums, part, total;   // byte offsets
};

bool small_weight_tiles(const mace_linear_desc& d) {
  return ceil_div(d.n_in, 128) * ceil_div(d.n_out, 128) * d.n_groups * std::max<int64_t>(1, d.n_rows / d.n_groups / 512) < kFillBlocks;
}

BackwardPlan plan_backward(const mace_linear_desc& d, bool bias, bool weights) {
  BackwardPlan p{};
  const int b = small_weight_tiles(d) ? 64 : 128;
  p.splits = weight_splits(d, b, b);
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

template <class T> struct Shapes {
  using Mid = TileShape<128, 128, 2, 2, 64, 2>;
  using Small = TileShape<64, 64, 2, 2, 64, 2>;
};
template <> struct Shapes<float> {
  using Mid = TileShape<128, 128, 2, 2, 32, 1>;
  using Small = TileShape<64, 64, 2, 2, 32, 1>;
};

mace_status launched() { return hipGetLastError() == hipSuccess ? MACE_OK : MACE_EHIP; }

template <class T>
mace_status forward(const mace_linear_desc& d, const void* x, const void* w, const void* bias, const void* residual,
                    const int* offsets, void* y, void* z, hipStream_t s) {
  LinearArgs<T> a{(const T*)x, (const T*)w, (const T*)bias, (const T*)residual, (T*)y, (T*)z, offsets, d.n_rows,
                  d.ld_x, d.ld_y, d.ld_residual, d.ld_preact, d.n_in, d.n_out, d.n_groups, d.act};
  const bool al = aligned16(x) && aligned16(w) && aligned16(bias) && aligned16(residual) && aligned16(y) &&
                  aligned16(z) && ((d.n_in | d.n_out | d.ld_x | d.ld_y | d.ld_residual | d.ld_preact) & 7) == 0;
  auto go = [&](auto shape) -> mace_status {
    using S = decltype(shape);
    const int64_t blocks = (ceil_div(d.n_rows, S::BM) + (offsets ? d.n_groups : 0)) * ceil_div(d.n_out, S::BN);
    if (blocks > INT32_MAX) return MACE_EUNSUPPORTED;
    if (al) linear_fwd_kernel<T, true, S><<<(unsigned)blocks, S::NT, 0, s>>>(a);
    else linear_fwd_kernel<T, false, S><<<(unsigned)blocks, S::NT, 0, s>>>(a);
    return launched();
  };
  using Mid = typename Shapes<T>::Mid;
  if (ceil_div(d.n_rows, Mid::BM) * ceil_div(d.n_out, Mid::BN) >= kFillBlocks) return go(Mid{});
  return go(typename Shapes<T>::Small{});
}

template <class T>
mace_status backward(const mace_linear_desc& d, const void* dy, int64_t lddy, const void* x, const void* w, const void* z,
                     const int* offsets, void* dx, int64_t lddx, void* dw, void* db, char* ws, hipStream_t s) {
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
    const bool al = aligned16(dy) && aligned16(z) && ((d.n_out | lddy | d.ld_preact) & 7) == 0;
    const dim3 grid((unsigned)slope_runs(d), (unsigned)ceil_div(vecs, cx));
    T* out = d.act != MACE_ACT_NONE ? const_cast<T*>(dz) : nullptr;
    auto go = [&](auto f) {
      f<<<grid, 256, 0, s>>>((const T*)dy, lddy, (const T*)z, d.ld_preact, out, lddz, db ? sums : nullptr, offsets,
                             d.n_groups, d.n_rows, d.n_out, d.act, slope_run(d.n_rows), cx);
    };
    if (al) go(linear_slope_kernel<T, true>);
    else go(linear_slope_kernel<T, false>);
    if ((st = launched()) != MACE_OK) return st;
  }
  const bool al_z = aligned16(dz) && ((d.n_in | d.n_out | lddz) & 7) == 0;
  const bool al_x = al_z && aligned16(w) && aligned16(dx) && (lddx & 7) == 0;
  const bool al_w = al_z && aligned16(x) && aligned16(dw) && (d.ld_x & 7) == 0;
  const RowGradArgs<T> ra{dz, (const T*)w, (T*)dx, offsets, d.n_rows, lddz, lddx, d.n_in, d.n_out, d.n_groups};
  const WeightGradArgs<T> wa{(const T*)x, dz, (T*)dw, p.splits > 1 ? reinterpret_cast<float*>(ws + p.part) : nullptr,
                             offsets, d.n_rows, d.ld_x, lddz, d.n_in, d.n_out, d.n_groups, p.splits};
  const BiasGradArgs<T> ba{sums, (T*)db, offsets, d.n_rows, d.n_out, slope_run(d.n_rows), (int)slope_runs(d)};
  auto go = [&](auto shape, bool rows, bool weights, bool bias) -> mace_status {
    using S = decltype(shape);
    static_assert(S::NT == 256, "bias_grad's lanes");
    const int64_t rb = rows ? (ceil_div(d.n_rows, S::BM) + (offsets ? d.n_groups : 0)) * ceil_div(d.n_in, S::BN) : 0;
    const int64_t wb = weights ? ceil_div(d.n_in, S::BM) * ceil_div(d.n_out, S::BN) * d.n_groups * p.splits : 0;
    const int64_t blocks = rb + wb + (bias ? ceil_div(d.n_out, 64) * d.n_groups : 0);
    if (blocks > INT32_MAX) return MACE_EUNSUPPORTED;
    if (blocks == 0) return MACE_OK;
    auto f = al_x && al_w ? linear_grad_kernel<T, true, true, S>
                          : (al_x ? linear_grad_kernel<T, true, false, S>
                                  : (al_w ? linear_grad_kernel<T, false, true, S> : linear_grad_kernel<T, false, false, S>));
    f<<<(unsigned)blocks, S::NT, 0, s>>>(ra, wa, ba, (int)rb, (int)wb);
    return launched();
  };
  using Mid = typename Shapes<T>::Mid;
  using Small = typename Shapes<T>::Small;
  const bool want_x = dx && d.n_rows > 0;
  const bool small_x = ceil_div(d.n_rows, Mid::BM) * ceil_div(d.n_in, Mid::BN) < kFillBlocks;
  const bool small_w = small_weight_tiles(d);
  const bool x_big = want_x && !small_x, w_big = dw && !small_w;
  if (x_big || w_big) {
    if ((st = go(Mid{}, x_big, w_big, db != nullptr)) != MACE_OK) return st;
    if ((st = go(Small{}, want_x && small_x, dw && small_w, false)) != MACE_OK) return st;
  } else {
    if ((st = go(Small{}, want_x, dw != nullptr, db != nullptr)) != MACE_OK) return st;
  }
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
  char* ws = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(workspace) + 255) & ~uintptr_t(255));
  if (p.total > 0 && size_t(ws - static_cast<char*>(workspace)) + p.total > workspace_bytes) return MACE_ENOSPACE;
  hipStream_t s = (hipStream_t)stream;
  if (d.dtype == MACE_TYPE_FP32)
    return backward<float>(d, dy, ld_dy, x, weights, preact, group_offsets, dx, ld_dx, dweights, dbias, ws, s);
  if (d.dtype == MACE_TYPE_BF16)
    return backward<__bf16>(d, dy, ld_dy, x, weights, preact, group_offsets, dx, ld_dx, dweights, dbias, ws, s);
  return backward<_Float16>(d, dy, ld_dy, x, weights, preact, group_offsets, dx, ld_dx, dweights, dbias, ws, s);
}
