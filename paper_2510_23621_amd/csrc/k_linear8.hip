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

// y = act(sx sw (qx qw) + b) + r: exact integer sums on v_mfma_i32_16x16x64_i8, through the
// tiles of the 16-bit layers, which move the same bytes per instruction.
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
  tile_gemm_direct<IntPair, S, true, true>({x, a.ldx, run.rows, 0}, {w, p.ldw, cols, 0}, a.n_in, lds, tid, acc);
  constexpr int W = lane_width<T>, NV = lane_vectors<S::TN, W>;
  const int l = tid & 63, wv = tid >> 6;
  const int m0 = (wv / S::WN) * (S::BM / S::WM) + (l & 15), n0 = (wv % S::WN) * (S::BN / S::WN);
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
  linear_epilogue<T, AL, S>(a, run, c0, cols, y, (T*)nullptr, tid, [&](int j, int i) {
    V v = lane_values<W>(acc, j, i);
#pragma unroll
    for (int q = 0; q < W; ++q) v[q] = (float)__float_as_int(v[q]) * xs[i] * ws[j][q];
    return v;
  });
}

// ------------------------------------------------------------------ host
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
size_t round256(size_t b) { return (b + 255) & ~size_t(255); }
int64_t padded(int n_in) { return ceil_div(n_in, 16) * 16; }
size_t size_of(int dtype) { return dtype == MACE_TYPE_FP32 ? 4 : 2; }

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

template <class F>
mace_status with_shape(int64_t rows, int64_t cols, int64_t groups, F f) {
  if ((groups == 1 || rows / groups >= 512) && ceil_div(rows, 256) * ceil_div(cols, 256) >= 192) return f(Large{});
  if (ceil_div(rows, 128) * ceil_div(cols, 128) >= 256) return f(Mid{});
  return f(Small{});
}

template <class T>
mace_status forward(const mace_linear_desc& d, const void* x8, int64_t ld_x8, const float* xs, const void* w8, int64_t ld_w,
                    const float* ws, const void* bias, const void* residual, const int* offsets, void* y, hipStream_t s) {
  const Linear8Args<T> p{{(const T*)x8, (const T*)w8, (const T*)bias, (const T*)residual, (T*)y, nullptr, offsets, d.n_rows,
                          ld_x8 / 2, d.ld_y, d.ld_residual, d.ld_y, (int)padded(d.n_in) / 2, d.n_out, d.n_groups, d.act},
                         xs, ws, ld_w / 2};
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
  if (!x_scales) {
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
