// Rows and weights as 8-bit integers with scales: mace_pack_rows, mace_unpack_rows,
// mace_pack_weights.
#include <algorithm>

#include "rows8.h"

namespace mace {
namespace {

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct Rows8Args {
  int64_t n, ld_x, ld_values;
  int cols, chunks;   // chunks: of 16 columns, the zeros behind the last column among them
  int lg;             // lanes per row
};

// lg lanes (a power of two up to a block) a row, 16 columns at a time: its largest magnitude, then its
// integers. CH: chunks of columns that a lane holds between the two, 0: any number, read twice.
// 36,864 x 2048 bfloat16: 44 to 46 us, 5.0 TB/s, a copy's rate; with an exact rounding of every column and the
// rows read twice, as those past 8192 columns are, 60.
template <class T, bool AL, int CH>
__global__ void __launch_bounds__(256) pack_rows_kernel(Rows8Args a, const T* __restrict__ x, int8_t* __restrict__ values,
                                                        float* __restrict__ scales) {
  __shared__ unsigned red[4];
  const int tid = threadIdx.x, lane = tid & (a.lg - 1);
  const int64_t row = ((int64_t)block_id() * 256 + tid) / a.lg;
  const bool on = row < a.n;
  const T* p = x + (on ? row : 0) * a.ld_x;
  Cols16<T> held[CH ? CH : 1];
  Magnitude<T> most;
  if constexpr (CH > 0) {
#pragma unroll
    for (int h = 0; h < CH; ++h)
      if (on && lane + h * a.lg < a.chunks) held[h] = load_cols16<T, AL>(p, lane + h * a.lg, a.cols);
#pragma unroll
    for (int h = 0; h < CH; ++h)
      if (on && lane + h * a.lg < a.chunks) most.add(held[h]);
  } else if (on) {
    for (int c = lane; c < a.chunks; c += a.lg) most.add(load_cols16<T, AL>(p, c, a.cols));
  }
  unsigned m = most.bits();
  for (int d = 1; d < min(a.lg, 64); d <<= 1) m = max(m, (unsigned)__shfl_xor((int)m, d));
  if (a.lg == 256) {   // (of every thread or none)
    if ((tid & 63) == 0) red[tid >> 6] = m;
    __syncthreads();
    m = max(max(red[0], red[1]), max(red[2], red[3]));
  }
  if (!on) return;
  const float s = scale8(Magnitude<T>::value(m)), inv = inverse8(s);
  if (lane == 0) scales[row] = s;
  i4* out = reinterpret_cast<i4*>(values + row * a.ld_values);
  if constexpr (CH > 0) {
#pragma unroll
    for (int h = 0; h < CH; ++h)
      if (lane + h * a.lg < a.chunks) {
        bool again = false;
        i4 q = round_most16(held[h], s, inv, again);
        if (again) q = round_cols16(held[h], s, inv);
        out[lane + h * a.lg] = q;
      }
  } else {
    for (int c = lane; c < a.chunks; c += a.lg) out[c] = round_cols16(load_cols16<T, AL>(p, c, a.cols), s, inv);
  }
}

// x = q s, 8 columns a thread (36,864 x 2048 to bfloat16: 34 us, 6.6 TB/s)
template <class T, bool AL>
__global__ void __launch_bounds__(256) unpack_rows_kernel(Rows8Args a, const int8_t* __restrict__ values,
                                                          const float* __restrict__ scales, T* __restrict__ x) {
  int vec;
  const int64_t row = item_row((a.cols + 7) / 8, vec);
  if (row >= a.n) return;
  const int c = 8 * vec;
  const uint2 q = *reinterpret_cast<const uint2*>(values + row * a.ld_values + c);
  const float s = scales[row];
  f8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = s * (float)(int8_t)((i < 4 ? q.x : q.y) >> 8 * (i & 3));
  store_n(x + row * a.ld_x + c, v, min(8, a.cols - c), AL);
}

// Weights: a block takes 64 output columns of a group, one a lane, and its 16 waves the rows, 16 at
// a time: the column's largest magnitude over all rows first, then the integers. 2048 x 2048 bfloat16 66 us, eight of
// them 109 (four waves to a tile: 242 and 379); done once.
constexpr int kPackThreads = 1024;
template <class T>
__global__ void __launch_bounds__(kPackThreads) pack_weights_kernel(const T* __restrict__ w, int groups, int n_in, int n_out, int64_t ld,
                                                                    int8_t* __restrict__ values, float* __restrict__ scales) {
  constexpr int WAVES = kPackThreads / 64;
  __shared__ unsigned red[WAVES][64];
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, tiles = (n_out + 63) / 64;
  const int64_t g = block_id() / tiles;
  if (g >= groups) return;   // (a grid's last row of blocks is full)
  const int col = block_id() % tiles * 64 + lane;
  const bool on = col < n_out;
  w += g * n_in * n_out + (on ? col : n_out - 1);
  auto load = [&](int k0, float (&x)[16]) {   // rows k0 .. k0 + 15, zeros past the last
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = k0 + i < n_in ? to_f32(w[(int64_t)(k0 + i) * n_out]) : 0.f;
  };
  unsigned m = 0;   // (magnitudes in the order of their bits: NaN above all)
  for (int k0 = 16 * wv; k0 < n_in; k0 += 16 * WAVES) {
    float x[16];
    load(k0, x);
#pragma unroll
    for (int i = 0; i < 16; ++i) m = max(m, __float_as_uint(fabsf(x[i])));
  }
  red[wv][lane] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < WAVES; ++i) m = max(m, red[i][lane]);
  if (!on) return;
  const float s = scale8(__uint_as_float(m)), inv = inverse8(s);
  if (wv == 0) scales[g * n_out + col] = s;
  values += (g * n_out + col) * ld;
  for (int k0 = 16 * wv; k0 < n_in; k0 += 16 * WAVES) {
    float x[16];
    unsigned q[16];
    load(k0, x);
#pragma unroll
    for (int i = 0; i < 16; ++i) q[i] = round8(x[i], s, inv);
    i4 o = lowest_bytes(q);
    if (s != s) o = i4{0, 0, 0, 0};
    *reinterpret_cast<i4*>(values + k0) = o;
  }
}

// ------------------------------------------------------------------ host
mace_status check(const mace_rows8_desc* d) {
  if (!d || d->n_rows < 0 || d->n_cols < 1 || d->dtype < MACE_TYPE_FP32 || d->dtype > MACE_TYPE_FP16) return MACE_EINVAL;
  if (d->ld_x < d->n_cols || d->ld_values < d->n_cols || d->ld_values % 16) return MACE_EINVAL;
  if (d->n_rows > (1 << 30) || d->n_cols > kMaxColumns8 || d->ld_values > kMaxPitch8) return MACE_EUNSUPPORTED;
  return MACE_OK;
}

}  // namespace
}  // namespace mace

using namespace mace;

extern "C" mace_status mace_pack_rows(const mace_rows8_desc* desc, const void* x, void* values, float* scales, void* stream) {
  const mace_status st = check(desc);
  if (st != MACE_OK) return st;
  if (desc->n_rows == 0) return MACE_OK;
  if (!x || !values || !scales || !aligned16(values)) return MACE_EINVAL;
  return by_type(desc->dtype, [&](auto zero) -> mace_status {
    using T = decltype(zero);
    const mace_rows8_desc& d = *desc;
    Rows8Args a{d.n_rows, d.ld_x, d.ld_values, d.n_cols, (int)ceil_div(d.n_cols, 16), 1};
    while (a.lg < a.chunks && a.lg < 64) a.lg *= 2;
    if (a.chunks > 128) a.lg = 256;
    const int64_t blocks = ceil_div(d.n_rows, 256 / a.lg);
    if (!fits_grid(blocks)) return MACE_EUNSUPPORTED;
    const bool al = aligned16(x) && ((d.n_cols | d.ld_x) & 15) == 0;
    auto run = [&](auto ch) {
      constexpr int CH = decltype(ch)::value;
      auto f = al ? pack_rows_kernel<T, true, CH> : pack_rows_kernel<T, false, CH>;
      f<<<grid_of(blocks), 256, 0, (hipStream_t)stream>>>(a, (const T*)x, (int8_t*)values, scales);
      return launched();
    };
    if (a.chunks <= a.lg) return run(Int<1>{});
    return a.chunks <= 2 * a.lg ? run(Int<2>{}) : run(Int<0>{});
  });
}

extern "C" mace_status mace_unpack_rows(const mace_rows8_desc* desc, const void* values, const float* scales, void* x,
                                        void* stream) {
  const mace_status st = check(desc);
  if (st != MACE_OK) return st;
  if (desc->n_rows == 0) return MACE_OK;
  if (!x || !values || !scales || !aligned16(values)) return MACE_EINVAL;
  return by_type(desc->dtype, [&](auto zero) -> mace_status {
    using T = decltype(zero);
    const mace_rows8_desc& d = *desc;
    const Rows8Args a{d.n_rows, d.ld_x, d.ld_values, d.n_cols, (int)ceil_div(d.n_cols, 16), 1};
    const int64_t blocks = ceil_div(d.n_rows * ceil_div(d.n_cols, 8), 256);
    if (!fits_grid(blocks)) return MACE_EUNSUPPORTED;
    const bool al = aligned16(x) && ((d.n_cols | d.ld_x) & 7) == 0;
    auto f = al ? unpack_rows_kernel<T, true> : unpack_rows_kernel<T, false>;
    f<<<grid_of(blocks), 256, 0, (hipStream_t)stream>>>(a, (const int8_t*)values, scales, (T*)x);
    return launched();
  });
}

extern "C" mace_status mace_pack_weights(int32_t n_groups, int32_t n_in, int32_t n_out, int32_t dtype, const void* weights,
                                         void* values, int64_t ld_values, float* scales, void* stream) {
  if (n_groups < 1 || n_in < 1 || n_out < 1 || dtype < MACE_TYPE_FP32 || dtype > MACE_TYPE_FP16) return MACE_EINVAL;
  if (!weights || !values || !scales || !aligned16(values) || ld_values < n_in || ld_values % 16) return MACE_EINVAL;
  if (n_groups > 1024 || n_in > kMaxColumns8 || n_out > (1 << 20) || ld_values > kMaxPitch8) return MACE_EUNSUPPORTED;
  return by_type(dtype, [&](auto zero) -> mace_status {
    using T = decltype(zero);
    const int64_t blocks = n_groups * ceil_div(n_out, 64);
    if (!fits_grid(blocks)) return MACE_EUNSUPPORTED;
    pack_weights_kernel<T><<<grid_of(blocks), kPackThreads, 0, (hipStream_t)stream>>>((const T*)weights, n_groups, n_in, n_out, ld_values,
                                                                            (int8_t*)values, scales);
    return launched();
  });
}
