// Embedding lookup and the gradient of its table: mace_embed_forward,
// mace_embed_backward.
#include <cmath>

#include "rows.h"
#include "sort.h"

namespace mace {
namespace {

struct EmbedArgs {
  int64_t n, rows, ld_table, ld_out;
  int width, nv;   // nv: vectors of 16 bytes per row
  float scale;
};

// out[t] = scale table[ids[t]], a thread per 16 bytes of the result.
template <class T, bool AL>
__global__ void __launch_bounds__(256) embed_kernel(EmbedArgs a, const T* __restrict__ table, const int* __restrict__ ids,
                                                    T* __restrict__ out) {
  constexpr int VE = kVecElems<T>;
  int vec;
  const int64_t t = item_row(a.nv, vec);
  if (t >= a.n) return;
  const int c = vec * VE, n = a.width - c, id = ids[t];
  RowVec<T> v;
  if (id >= 0 && id < a.rows) {
    v = load_vec<T, AL>(table + id * a.ld_table + c, n);
#pragma unroll
    for (int q = 0; q < VE; ++q) v.e[q] = (T)(a.scale * to_f32(v.e[q]));
  } else {
#pragma unroll
    for (int q = 0; q < VE; ++q) v.e[q] = (T)0.f;
  }
  store_vec<T, AL>(out + t * a.ld_out + c, v, n);
}

// One pass of the sort by id, lowest digit first: ids outside the table count as
// `rows`, behind all others. The first pass has no slots yet: they are 0, 1, ...
struct EmbedSlots {
  const int *key_in, *slot_in;
  int *key_out, *slot_out;
  int rows, shift, mask;
  __device__ __forceinline__ int key(int64_t s) const {
    const int k = key_in[s];
    return k >= 0 && k < rows ? k : rows;
  }
  __device__ __forceinline__ int bucket(int64_t s) const { return key(s) >> shift & mask; }
  __device__ __forceinline__ void place(int64_t s, int row) const {
    key_out[row] = key(s);
    slot_out[row] = slot_in ? slot_in[s] : (int)s;
  }
};

struct EmbedGradArgs {
  int64_t n, ld_dout, ld_table;
  int rows, width, nv, lg, seg;   // lg lanes share a segment's row, seg sorted slots per segment
  int64_t segments;
  float scale;
  const int *key, *slot;   // sorted
  float* part;             // [segments][2][width]
};

// Sums over the sorted slots. lg lanes (a power of two) take a segment of them and
// 16 bytes of the columns each, and add the rows of dout in their order; a run of equal ids
// that lies within the segment goes to the table, the parts of one that was begun
// before (0) or goes on behind (1; also where it begins at the segment's first slot)
// to part, for the join.
template <class T, bool AL>
__global__ void __launch_bounds__(256) embed_sum_kernel(EmbedGradArgs a, const T* __restrict__ dout, T* __restrict__ dtable) {
  constexpr int VE = kVecElems<T>, U = 8;
  const int64_t seg = ((int64_t)block_id() * 256 + threadIdx.x) / a.lg;
  if (seg >= a.segments) return;
  const int64_t r0 = seg * a.seg, r1 = min<int64_t>(a.n, r0 + a.seg);
  const int before = r0 > 0 ? a.key[r0 - 1] : -1, after = r1 < a.n ? a.key[r1] : -1;
  for (int vec = threadIdx.x & (a.lg - 1); vec < a.nv; vec += a.lg) {
    const int c = vec * VE, n = a.width - c;
    float acc[VE] = {};
    int key = a.key[r0];
    bool begun = key == before;
    auto flush = [&](bool goes_on) {
      if (key >= a.rows) return;
      if (begun || goes_on) {
        float* p = a.part + (2 * seg + (begun ? 0 : 1)) * a.width + c;
#pragma unroll
        for (int q = 0; q < VE; ++q)
          if (q < n) p[q] = acc[q];
      } else {
        RowVec<T> o;
#pragma unroll
        for (int q = 0; q < VE; ++q) o.e[q] = (T)(a.scale * acc[q]);
        store_vec<T, AL>(dtable + key * a.ld_table + c, o, n);
      }
    };
    for (int64_t r = r0; r < r1; r += U) {
      int k[U];
      RowVec<T> v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t s = min(r + u, r1 - 1);
        k[u] = a.key[s];
        if (k[u] < a.rows) v[u] = load_vec<T, AL>(dout + a.slot[s] * a.ld_dout + c, n);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (r + u >= r1) continue;
        if (k[u] != key) {
          flush(false);
          key = k[u];
          begun = false;
#pragma unroll
          for (int q = 0; q < VE; ++q) acc[q] = 0.f;
        }
        if (k[u] < a.rows)
#pragma unroll
          for (int q = 0; q < VE; ++q) acc[q] += to_f32(v[u].e[q]);
      }
    }
    flush(key == after);
  }
}

// first sorted slot with a key of at least v
__device__ __forceinline__ int64_t lower_bound(const int* __restrict__ key, int64_t n, int v) {
  int64_t lo = 0, hi = n;
  while (lo < hi) {
    const int64_t m = (lo + hi) >> 1;
    if (key[m] < v) lo = m + 1;
    else hi = m;
  }
  return lo;
}

// Zeros in the rows that no id names: a wave looks for 64 rows at a time, a lane each, and
// writes those that are missing.
template <class T, bool AL>
__global__ void __launch_bounds__(256) embed_zero_kernel(EmbedGradArgs a, T* __restrict__ dtable) {
  constexpr int VE = kVecElems<T>;
  const int lane = threadIdx.x & 63;
  const int64_t v0 = ((int64_t)block_id() * 4 + (threadIdx.x >> 6)) * 64;
  if (v0 >= a.rows) return;
  const int64_t v = v0 + lane;
  bool gone = false;
  if (v < a.rows) {
    const int64_t at = lower_bound(a.key, a.n, (int)v);
    gone = at >= a.n || a.key[at] != v;
  }
  RowVec<T> zero;
#pragma unroll
  for (int q = 0; q < VE; ++q) zero.e[q] = (T)0.f;
  for (unsigned long long m = __ballot(gone); m; m &= m - 1) {
    T* row = dtable + (v0 + __ffsll(m) - 1) * a.ld_table;
    for (int vec = lane; vec < a.nv; vec += 64) store_vec<T, AL>(row + vec * VE, zero, a.width - vec * VE);
  }
}

// Runs that cross segments: the block of the segment that a run begins in adds its
// parts, waves' shares in the order of the segments, and then the shares in order.
constexpr int kJoinWaves = 16;
template <class T>
__global__ void __launch_bounds__(64 * kJoinWaves) embed_join_kernel(EmbedGradArgs a, T* __restrict__ dtable) {
  __shared__ float red[kJoinWaves][64];
  const int64_t blocks_n = (a.width + 63) / 64;
  const int64_t seg = block_id() / blocks_n;
  if (seg >= a.segments) return;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int col = (int)(block_id() % blocks_n) * 64 + lane;
  const int64_t r0 = seg * a.seg, r1 = min<int64_t>(a.n, r0 + a.seg);
  if (r1 >= a.n) return;
  const int key = a.key[r1 - 1];
  if (key >= a.rows || a.key[r1] != key) return;                      // nothing goes on behind
  if (r0 > 0 && a.key[r0] == key && a.key[r0 - 1] == key) return;     // begun before this segment
  const int64_t end = lower_bound(a.key, a.n, key + 1);               // (the run's end)
  const int64_t last = (end - 1) / a.seg, parts = last - seg + 1;
  const int64_t per = (parts + kJoinWaves - 1) / kJoinWaves, p0 = w * per, p1 = min(parts, p0 + per);
  float s = 0.f;
  if (col < a.width)
    for (int64_t p = p0; p < p1; ++p) s += a.part[(2 * (seg + p) + (p == 0 ? 1 : 0)) * a.width + col];
  red[w][lane] = s;
  __syncthreads();
  if (w == 0 && col < a.width) {
    for (int i = 1; i < kJoinWaves; ++i) s += red[i][lane];
    dtable[key * a.ld_table + col] = (T)(a.scale * s);
  }
}

// ------------------------------------------------------------------ host
mace_status check(const mace_embed_desc* d) {
  if (!d || d->n_ids < 0 || d->n_rows < 1 || d->width < 1) return MACE_EINVAL;
  if (d->dtype < MACE_TYPE_FP32 || d->dtype > MACE_TYPE_FP16 || !std::isfinite((float)d->scale)) return MACE_EINVAL;
  if (d->ld_table < d->width || d->ld_out < d->width) return MACE_EINVAL;
  if (d->n_ids > (1 << 30) || d->n_rows > (1 << 30) || d->width > (1 << 20)) return MACE_EUNSUPPORTED;
  return MACE_OK;
}
template <class T>
bool aligned(const mace_embed_desc& d, const void* a, const void* b) {
  const int ve = kVecElems<T>;
  return aligned16(a) && aligned16(b) && d.width % ve == 0 && d.ld_table % ve == 0 && d.ld_out % ve == 0;
}
size_t round256(size_t b) { return (b + 255) & ~size_t(255); }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Digits of the sort: ids and the number behind them, at most nine bits a pass.
struct SortPlan {
  int passes, bits;
  int buckets() const { return 1 << bits; }
};
SortPlan sort_plan(int64_t rows) {
  int bits = 1;
  while (int64_t(1) << bits <= rows) ++bits;
  const int passes = (bits + 8) / 9;
  return {passes, (bits + passes - 1) / passes};
}
constexpr int kSegment = 64;

struct BackwardPlan {
  SortPlan sort;
  int64_t segments;
  size_t hist, key[2], slot[2], part, total;
};
BackwardPlan plan_backward(const mace_embed_desc& d) {
  BackwardPlan p{};
  p.sort = sort_plan(d.n_rows);
  p.segments = ceil_div(d.n_ids, kSegment);
  size_t o = 0;
  auto take = [&](size_t bytes) {
    const size_t at = o;
    o += round256(bytes);
    return at;
  };
  p.hist = take(size_t(sort_blocks(d.n_ids)) * (p.sort.buckets() + 1) * sizeof(int));
  for (int i = 0; i < 2; ++i) {
    p.key[i] = take(size_t(d.n_ids) * sizeof(int));
    p.slot[i] = take(size_t(d.n_ids) * sizeof(int));
  }
  p.part = take(size_t(p.segments) * 2 * d.width * sizeof(float));
  p.total = o;
  return p;
}

}  // namespace
}  // namespace mace

using namespace mace;

extern "C" mace_status mace_embed_forward(const mace_embed_desc* desc, const void* table, const int32_t* ids, void* out,
                                          void* stream) {
  const mace_status st = check(desc);
  if (st != MACE_OK) return st;
  if (desc->n_ids == 0) return MACE_OK;
  if (!table || !ids || !out) return MACE_EINVAL;
  return by_type(desc->dtype, [&](auto zero) {
    using T = decltype(zero);
    const mace_embed_desc& d = *desc;
    const EmbedArgs a{d.n_ids, d.n_rows, d.ld_table, d.ld_out, d.width, (int)ceil_div(d.width, kVecElems<T>), (float)d.scale};
    const int64_t blocks = ceil_div(a.n * a.nv, 256);
    if (!fits_grid(blocks)) return MACE_EUNSUPPORTED;
    auto f = aligned<T>(d, table, out) ? embed_kernel<T, true> : embed_kernel<T, false>;
    f<<<grid_of(blocks), 256, 0, (hipStream_t)stream>>>(a, (const T*)table, ids, (T*)out);
    return launched();
  });
}

extern "C" size_t mace_embed_backward_workspace_bytes(const mace_embed_desc* desc) {
  if (check(desc) != MACE_OK) return 0;
  return plan_backward(*desc).total + 256;
}

extern "C" mace_status mace_embed_backward(const mace_embed_desc* desc, const void* dout, const int32_t* ids, void* dtable,
                                           void* workspace, size_t workspace_bytes, void* stream) {
  mace_status st = check(desc);
  if (st != MACE_OK) return st;
  if (!dtable || (desc->n_ids > 0 && (!dout || !ids || !workspace))) return MACE_EINVAL;
  const mace_embed_desc& d = *desc;
  const BackwardPlan p = plan_backward(d);
  if (d.n_ids > 0 && workspace_bytes < p.total + 256) return MACE_ENOSPACE;
  char* ws = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(workspace) + 255) & ~uintptr_t(255));
  auto ints = [&](size_t at) { return reinterpret_cast<int*>(ws + at); };
  hipStream_t s = (hipStream_t)stream;
  return by_type(d.dtype, [&](auto zero) -> mace_status {
    using T = decltype(zero);
    EmbedGradArgs a{};
    a.n = d.n_ids, a.ld_dout = d.ld_out, a.ld_table = d.ld_table, a.rows = (int)d.n_rows, a.width = d.width;
    a.nv = (int)ceil_div(d.width, kVecElems<T>), a.seg = kSegment, a.segments = p.segments, a.scale = (float)d.scale;
    a.lg = 1;
    while (a.lg < 64 && a.lg < a.nv) a.lg *= 2;
    a.part = reinterpret_cast<float*>(ws + p.part);
    const int64_t zero_blocks = ceil_div(d.n_rows, 256), sum_blocks = ceil_div(a.segments * a.lg, 256);
    const int64_t join_blocks = a.segments * ceil_div(d.width, 64);
    if (!fits_grid(zero_blocks) || !fits_grid(sum_blocks) || !fits_grid(join_blocks)) return MACE_EUNSUPPORTED;
    for (int i = 0; i < p.sort.passes && d.n_ids > 0; ++i) {
      const EmbedSlots sl{i ? ints(p.key[(i + 1) & 1]) : ids, i ? ints(p.slot[(i + 1) & 1]) : nullptr, ints(p.key[i & 1]),
                          ints(p.slot[i & 1]), a.rows, i * p.sort.bits, p.sort.buckets() - 1};
      const mace_status e = sort_slots(sl, d.n_ids, p.sort.buckets() - 1, ints(p.hist), nullptr, s);
      if (e != MACE_OK) return e;
    }
    a.key = ints(p.key[(p.sort.passes + 1) & 1]), a.slot = ints(p.slot[(p.sort.passes + 1) & 1]);
    const bool al = aligned<T>(d, dout, dtable);
    auto fz = al ? embed_zero_kernel<T, true> : embed_zero_kernel<T, false>;
    fz<<<grid_of(zero_blocks), 256, 0, s>>>(a, (T*)dtable);
    if ((st = launched()) != MACE_OK || d.n_ids == 0) return st;
    auto fs = al ? embed_sum_kernel<T, true> : embed_sum_kernel<T, false>;
    fs<<<grid_of(sum_blocks), 256, 0, s>>>(a, (const T*)dout, (T*)dtable);
    if ((st = launched()) != MACE_OK) return st;
    embed_join_kernel<T><<<grid_of(join_blocks), 64 * kJoinWaves, 0, s>>>(a, (T*)dtable);
    return launched();
  });
}
