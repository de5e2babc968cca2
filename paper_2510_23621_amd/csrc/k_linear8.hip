// Grouped dense layer on 8-bit rows and weights: mace_linear8_forward.
#include <algorithm>

#include "linear.h"
#include "rows8.h"

namespace mace {
namespace {

template <class T>
struct Linear8Args {
  LinearArgs<T> a;   // (x and w: the integers; ldx and n_in in pairs of them)
  const float *xs, *ws;
  int64_t ldw;   // in pairs
};

// sum sx sw + b for an integer sum (below 2^31). Its product with sx stays within FP32 up to 2^96; in a row
// with a larger scale (`large`) the smaller of the two scales comes first, so that no
// product is out of range unless the last one is. (Scales in the order of their bits, NaN last.)
constexpr float kLargeScale8 = 79228162514264337593543950336.f;   // 2^96
__device__ __forceinline__ float scaled8(int sum, float sx, float sw, float b, bool large) {
  float lo = sx, hi = sw;
  if (large) {
    lo = __int_as_float(min(__float_as_int(sx), __float_as_int(sw)));
    hi = __int_as_float(max(__float_as_int(sx), __float_as_int(sw)));
  }
  return __builtin_fmaf((float)sum * lo, hi, b);
}

// y = act(sx sw (qx qw) + b) + r: exact integer sums on v_mfma_i32_16x16x64_i8, through the
// tiles of the 16-bit layers, which move the same bytes per instruction. 36864 x 2048 x 2048 in eight groups to
// bfloat16, in a captured graph: 151 us bare (2.05 POP/s, where a library product of that size reaches 1.65 and a
// larger one 2.14), 210 with bias, SiLU and residual, whose 151 MB more and vector instructions come after the products:
// one block per CU, and nothing to run beside (one call at a time 235). Tiles of 128 x 128, of which two blocks fit, take
// 189 and 250. Residuals four tile rows ahead: one ahead 217 us, all eight 213.
template <class T, bool AL, class S>
__global__ void __launch_bounds__(S::NT) linear8_kernel(Linear8Args<T> p) {
  __shared__ __align__(16) unsigned short lds[tile_lds<IntPair, S>];
  const LinearArgs<T>& a = p.a;
  const int tid = threadIdx.x;
  const int tiles_n = (a.n_out + S::BN - 1) / S::BN;
  const int id = xcd_order(block_id(), block_count());
  const int c0 = id % tiles_n * S::BN, cols = min(S::BN, a.n_out - c0);
  RowRun run;
  if (!find_run(a.offsets, a.groups, a.n, S::BM, id / tiles_n, run)) return;
  T* y = a.y + run.row0 * a.ldy + c0;
  if (run.group >= a.groups) {
    zero_rows(y, a.ldy, run.rows, cols, tid, S::NT);
    return;
  }
  const int64_t w_row = (int64_t)run.group * a.n_out + c0;
  f4 acc[S::TN][S::TM];
  const IntPair *x = reinterpret_cast<const IntPair*>(a.x) + run.row0 * a.ldx;
  const IntPair *w = reinterpret_cast<const IntPair*>(a.w) + w_row * p.ldw;
  const int l = tid & 63, wv = tid >> 6;
  // the wave's rows' scales, whether one is large: requested before the products, and two forms of the
  // results (a branch for every row's values, or on scales requested after the products: 265 us where this takes 251)
  constexpr int WR = S::BM / S::WM;
  float row_scale[(WR + 63) / 64];
#pragma unroll
  for (int i = 0; i < (WR + 63) / 64; ++i)
    row_scale[i] = p.xs[run.row0 + min(wv / S::WN * WR + min(64 * i + l, WR - 1), run.rows - 1)];
  tile_gemm_direct<IntPair, S, true, true>({x, a.ldx, run.rows, 0}, {w, p.ldw, cols, 0}, a.n_in, lds, tid, acc);
  constexpr int W = lane_width<T>, NV = lane_vectors<S::TN, W>;
  bool large = false;
#pragma unroll
  for (float s : row_scale) large |= !(s <= kLargeScale8);
  const int m0 = (wv / S::WN) * WR + (l & 15), n0 = (wv % S::WN) * (S::BN / S::WN);
  using V = typename Floats<W>::type;
  float xs[S::TM];
  V ws[NV];
#pragma unroll
  for (int i = 0; i < S::TM; ++i) xs[i] = p.xs[run.row0 + min(m0 + 16 * i, run.rows - 1)];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int n = n0 + lane_column<W>(j, l);
    ws[j] = V{};
    if (n < cols) ws[j] = read_n<W>(p.ws + w_row + n, min(W, cols - n), false);
  }
  auto finish = [&](auto any_large) {
    linear_epilogue<T, AL, S, sizeof(T) == 2 ? 4 : 2, sizeof(T) == 2>(a, run, c0, cols, y, (T*)nullptr, tid, [&](int j, int i, V b) {
      V v = lane_values<W>(acc, j, i);
#pragma unroll
      for (int q = 0; q < W; ++q) v[q] = scaled8(__float_as_int(v[q]), xs[i], ws[j][q], b[q], any_large.value && !(xs[i] <= kLargeScale8));
      return v;
    });
  };
  if (__any(large)) finish(Int<1>{});
  else finish(Int<0>{});
}

// Few rows: a block of four waves forms 16 x 16 results, each wave a quarter of K, added through LDS.
// The rows lie in LDS as integers over all of K; where they come as T the block rounds them itself
// (no launch and no way through memory for them). The weights go straight to the matrix
// instructions, requested before the rows. One row of 2048 bfloat16 on 2048 x 2048: 6.0 to 7.2 us, of
// which the weights' 4 MB take 0.8 at a copy's rate; the rest is the launch and three dependent trips to memory.
constexpr int kThinRows = 16, kThinCols = 16, kThinLds = 56 << 10;
// bytes from row to row: 16 more than a multiple of 128, so that eight rows' 16 bytes lie in all banks
int thin_pitch(int n_in) { return (n_in + 127) / 128 * 128 + 16; }
int thin_rows(int64_t n) {   // that a block holds: a power of two of them
  int r = 1;
  while (r < n && r < kThinRows) r *= 2;
  return r;
}
int64_t thin_lds(const mace_linear_desc& d) { return (int64_t)thin_rows(d.n_rows) * thin_pitch(d.n_in); }

template <class T, bool AL, bool PACKED>
__global__ void __launch_bounds__(256) linear8_thin_kernel(Linear8Args<T> p, int n_in, int pitch, int held) {
  extern __shared__ __align__(16) int8_t rows8[];
  __shared__ float scale[kThinRows];
  __shared__ unsigned red[4];
  __shared__ i4 part[4 * 64];
  const LinearArgs<T>& a = p.a;
  const int tid = threadIdx.x, l = tid & 63, wv = tid >> 6, i = l & 15, g = l >> 4;
  const int tiles_n = (a.n_out + kThinCols - 1) / kThinCols;
  const int id = block_id();
  const int c0 = id % tiles_n * kThinCols, cols = min(kThinCols, a.n_out - c0);
  RowRun run;
  if (!find_run(a.offsets, a.groups, a.n, kThinRows, id / tiles_n, run)) return;
  T* y = a.y + run.row0 * a.ldy + c0;
  if (run.group >= a.groups) {
    zero_rows(y, a.ldy, run.rows, cols, tid, 256);
    return;
  }
  const int k16 = (n_in + 15) / 16 * 16;
  const int64_t w_row = (int64_t)run.group * a.n_out + c0;
  const int8_t* w = reinterpret_cast<const int8_t*>(a.w) + (w_row + min(i, cols - 1)) * 2 * p.ldw + 16 * g;
  constexpr int U = 8;   // steps of 64 products' indices in flight
  i4 wr[U];
  auto weights = [&](int at) {
    i4 q = {0, 0, 0, 0};
    if (at + 16 * g < k16) q = *reinterpret_cast<const i4*>(w + at);
    return q;
  };
#pragma unroll
  for (int u = 0; u < U; ++u) wr[u] = weights(64 * wv + 256 * u);
  // what the epilogue adds, requested before the rows too
  const int n = 4 * g, count = min(4, cols - n);
  typedef T t4 __attribute__((ext_vector_type(4)));
  t4 res = {};
  f4 ws = {0.f, 0.f, 0.f, 0.f}, bias = ws;
  if (wv == 0 && count > 0) {
    ws = read_n<4>(p.ws + w_row + n, count, false);
    if (a.bias) bias = read_n<4>(a.bias + w_row + n, count, false);
    if (a.residual && i < run.rows) res = read_raw<4>(a.residual + (run.row0 + i) * a.ldr + c0 + n, count, false);
  }
  // rows: tpr threads (a power of two) each, 16 columns at a time, zeros from k16 on
  int tpr = 256 / kThinRows;
  while (tpr < 256 && 256 / (2 * tpr) >= run.rows) tpr *= 2;
  const int row = tid / tpr, t = tid & (tpr - 1), chunks = pitch / 16 - 1;
  const int64_t r = run.row0 + min(row, run.rows - 1);
  int8_t* mine = rows8 + row * pitch;
  if constexpr (PACKED) {
    const int8_t* x = reinterpret_cast<const int8_t*>(a.x) + r * 2 * a.ldx;
    for (int c = t; c < chunks; c += tpr) {
      i4 q = {0, 0, 0, 0};
      if (16 * c < k16) q = *reinterpret_cast<const i4*>(x + 16 * c);
      *reinterpret_cast<i4*>(mine + 16 * c) = q;
    }
    if (t == 0) scale[row] = p.xs[r];
  } else {
    const T* x = a.x + r * a.ldx;
    constexpr int H = sizeof(T) == 2 ? 8 : 4;   // chunks requested at a time; the first ones stay in registers
    Cols16<T> v[H];
    auto load = [&](int c) {
#pragma unroll
      for (int h = 0; h < H; ++h)
        if (16 * (c + h * tpr) < n_in) v[h] = load_cols16<T, AL>(x, c + h * tpr, n_in);
    };
    Magnitude<T> most;
    for (int c = t + H * tpr * ((chunks - 1 - t) / (H * tpr)); c >= 0; c -= H * tpr) {   // (the first ones last)
      load(c);
#pragma unroll
      for (int h = 0; h < H; ++h)
        if (16 * (c + h * tpr) < n_in) most.add(v[h]);
    }
    unsigned m = most.bits();
    for (int d = 1; d < min(tpr, 64); d <<= 1) m = max(m, (unsigned)__shfl_xor((int)m, d));
    if (tpr > 64) {   // (of every thread or none)
      if (l == 0) red[wv] = m;
      __syncthreads();
      for (int q = 0; q < tpr / 64; ++q) m = max(m, red[row * (tpr / 64) + q]);
    }
    const float s = scale8(Magnitude<T>::value(m)), inv = inverse8(s);
    bool again = false;
    for (int c = t; c < chunks; c += H * tpr) {
      if (c > t) load(c);
#pragma unroll
      for (int h = 0; h < H; ++h)
        if (c + h * tpr < chunks) {
          i4 q = {0, 0, 0, 0};
          if (16 * (c + h * tpr) < n_in) q = round_most16(v[h], s, inv, again);
          *reinterpret_cast<i4*>(mine + 16 * (c + h * tpr)) = q;
        }
    }
    if (again)   // (apart, and one chunk at a time: a block runs through this code once, and waits for its instructions)
#pragma unroll 1
      for (int c = t; 16 * c < n_in; c += tpr)
        *reinterpret_cast<i4*>(mine + 16 * c) = round_cols16(load_cols16<T, AL>(x, c, n_in), s, inv);
    if (t == 0) scale[row] = s;
  }
  __syncthreads();
  // (rows past the run's are as LDS held them, or the last one's: integers, whose results are not stored)
  const int8_t* xr = rows8 + min(i, held - 1) * pitch + 16 * g;
  i4 acc = {0, 0, 0, 0};
  for (int k = 64 * wv; k < k16; k += 256 * U) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = k + 256 * u;
      if (at < k16) {
        acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(wr[u], *reinterpret_cast<const i4*>(xr + at), acc, 0, 0, 0);
        wr[u] = weights(at + 256 * U);
      }
    }
  }
  part[tid] = acc;
  __syncthreads();
  if (wv || count <= 0 || i >= run.rows) return;
  acc = (part[l] + part[64 + l]) + (part[128 + l] + part[192 + l]);
  f4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[e] = scaled8(acc[e], scale[i], ws[e], bias[e], !(scale[i] <= kLargeScale8));
    v[e] = a.act == MACE_ACT_SILU ? activate_as<MACE_ACT_SILU, sizeof(T) == 2>(v[e])
                                  : (a.act == MACE_ACT_GELU ? activate<MACE_ACT_GELU>(v[e]) : v[e]);
  }
  if (a.residual) v += __builtin_convertvector(res, f4);
  store_n(y + i * a.ldy + n, v, count, false);
}

// ------------------------------------------------------------------ host
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
size_t round256(size_t b) { return (b + 255) & ~size_t(255); }
int64_t padded(int n_in) { return ceil_div(n_in, 16) * 16; }

mace_status check(const mace_linear_desc* d) {
  if (!d || d->n_rows < 0 || d->n_in < 1 || d->n_out < 1 || d->n_groups < 1) return MACE_EINVAL;
  if (d->dtype < MACE_TYPE_FP32 || d->dtype > MACE_TYPE_FP16 || d->act < MACE_ACT_NONE || d->act > MACE_ACT_GELU)
    return MACE_EINVAL;
  if (d->ld_x < d->n_in || d->ld_y < d->n_out || d->ld_residual < d->n_out) return MACE_EINVAL;
  if (d->n_rows > (1 << 30) || d->n_in > kMaxColumns8 || d->n_out > (1 << 20) || d->n_groups > 1024) return MACE_EUNSUPPORTED;
  return MACE_OK;
}

using Large = TileShape<256, 256, 2, 4, 64, 2, true>;
using Mid = TileShape<128, 128, 2, 2, 64, 2, true>;
using Small = TileShape<64, 64, 2, 2, 64, 4, true>;

// Large from 192 blocks of its own on, of groups of 512 rows or more, Mid from 256: rows in 8 bits, SiLU and a
// residual, 8192 x 2048 x 2048 (256 Large) 40 us against 44 as Mid, 6144 rows (192) 39.7 against 38.7, with K = 4096 57
// against 60, 4096 rows (128) 35.8 against 24.4 (12288, a round and a half of Large, 71 against 66);
// 2048 x 2048 x 2048 (256 Mid) 18.6 against 21.3 as Small, 4096 x 512 x 512 (128) 9.1 against 5.9.
template <class F>
mace_status with_shape(int64_t rows, int64_t cols, int64_t groups, F f) {
  if ((groups == 1 || rows / groups >= 512) && ceil_div(rows, 256) * ceil_div(cols, 256) >= 192) return f(Large{});
  if (ceil_div(rows, 128) * ceil_div(cols, 128) >= 256) return f(Mid{});
  return f(Small{});
}

// The thin kernel up to two blocks per CU, where K fits LDS: rounding a block's rows again for every
// 16 columns costs it more on larger launches. With rows in bfloat16 (the other way rounds them in a
// launch of its own): 1 x 2048 x 2048 (128 blocks) 6.0 us against 10.0, 256 x 97 x 211 (224) 6.5
// against 8.8, 64 x 512 x 2048 (512) 7.4 against 7.6, 128 x 512 x 2048 (1024) 13.0 against 7.7.
constexpr int kThinBlocks = 512;
bool thin(const mace_linear_desc& d) {
  return thin_lds(d) <= kThinLds && ceil_div(d.n_rows, kThinRows) * ceil_div(d.n_out, kThinCols) <= kThinBlocks;
}
template <class T>
mace_status forward_thin(const mace_linear_desc& d, const Linear8Args<T>& p, bool packed, hipStream_t s) {
  const int64_t blocks = (ceil_div(d.n_rows, kThinRows) + (p.a.offsets ? d.n_groups : 0)) * ceil_div(d.n_out, kThinCols);
  if (!fits_grid(blocks)) return MACE_EUNSUPPORTED;
  const bool al = aligned16(p.a.x) && ((d.n_in | d.ld_x) & 15) == 0;
  auto f = packed ? linear8_thin_kernel<T, true, true>
                  : (al ? linear8_thin_kernel<T, true, false> : linear8_thin_kernel<T, false, false>);
  f<<<grid_of(blocks), 256, (unsigned)thin_lds(d), s>>>(p, d.n_in, thin_pitch(d.n_in), thin_rows(d.n_rows));
  return launched();
}

template <class T>
mace_status forward(const mace_linear_desc& d, const void* x8, int64_t ld_x8, const float* xs, const void* w8, int64_t ld_w,
                    const float* ws, const void* bias, const void* residual, const int* offsets, void* y, hipStream_t s) {
  const Linear8Args<T> p{{(const T*)x8, (const T*)w8, (const T*)bias, (const T*)residual, (T*)y, nullptr, offsets, d.n_rows,
                          xs ? ld_x8 / 2 : ld_x8, d.ld_y, d.ld_residual, d.ld_y, (int)padded(d.n_in) / 2, d.n_out, d.n_groups, d.act},
                         xs, ws, ld_w / 2};
  if (thin(d)) return forward_thin<T>(d, p, xs != nullptr, s);
  const bool al = aligned16(bias) && aligned16(residual) && aligned16(y) &&
                  ((d.n_out | d.ld_y | (residual ? d.ld_residual : 0)) & 7) == 0;
  return with_shape(d.n_rows, d.n_out, d.n_groups, [&](auto shape) -> mace_status {
    using S = decltype(shape);
    const int64_t blocks = (ceil_div(d.n_rows, S::BM) + (offsets ? d.n_groups : 0)) * ceil_div(d.n_out, S::BN);
    if (!fits_grid(blocks)) return MACE_EUNSUPPORTED;
    auto f = al ? linear8_kernel<T, true, S> : linear8_kernel<T, false, S>;
    f<<<grid_of(blocks), S::NT, 0, s>>>(p);
    return launched();
  });
}

}  // namespace
}  // namespace mace

using namespace mace;

extern "C" size_t mace_linear8_workspace_bytes(const mace_linear_desc* desc) {
  if (check(desc) != MACE_OK) return 0;
  if (thin(*desc)) return 256;
  return 256 + round256(size_t(desc->n_rows) * padded(desc->n_in)) + round256(size_t(desc->n_rows) * sizeof(float));
}

extern "C" mace_status mace_linear8_forward(const mace_linear_desc* desc, const void* x8, const float* x_scales,
                                            const void* w8, int64_t ld_w, const float* w_scales, const void* bias,
                                            const void* residual, const int32_t* group_offsets, void* y, void* workspace,
                                            size_t workspace_bytes, void* stream) {
  mace_status st = check(desc);
  if (st != MACE_OK) return st;
  const mace_linear_desc& d = *desc;
  if (!w8 || !w_scales || !aligned16(w8) || ld_w < d.n_in || ld_w % 16 || (d.n_groups > 1 && !group_offsets)) return MACE_EINVAL;
  if (d.n_rows > 0 && (!x8 || !y)) return MACE_EINVAL;
  if (x_scales && (d.ld_x % 16 || !aligned16(x8))) return MACE_EINVAL;
  if (ld_w > kMaxPitch8 || (x_scales && d.ld_x > kMaxPitch8)) return MACE_EUNSUPPORTED;
  if (d.n_rows == 0) return MACE_OK;
  int64_t ld = d.ld_x;
  if (!x_scales && !thin(d)) {
    if (!workspace) return MACE_EINVAL;
    if (workspace_bytes < mace_linear8_workspace_bytes(desc)) return MACE_ENOSPACE;
    char* ws = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(workspace) + 255) & ~uintptr_t(255));
    float* scales = reinterpret_cast<float*>(ws + round256(size_t(d.n_rows) * padded(d.n_in)));
    ld = padded(d.n_in);
    const mace_rows8_desc r{d.n_rows, d.n_in, d.dtype, d.ld_x, ld};
    if ((st = mace_pack_rows(&r, x8, ws, scales, stream)) != MACE_OK) return st;
    x8 = ws;
    x_scales = scales;
  }
  return by_type(d.dtype, [&](auto zero) {
    return forward<decltype(zero)>(d, x8, ld, x_scales, w8, ld_w, w_scales, bias, residual, group_offsets, y,
                                   (hipStream_t)stream);
  });
}
