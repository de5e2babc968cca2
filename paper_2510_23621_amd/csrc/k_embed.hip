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

// out[t] = scale table[ids[t]], a thread per 16 bytes of the result, U of them 256
// apart: their ids first, then their rows, then the stores. 131,072 rows of 1024 bfloat16 out of 32,000: 74 us,
// 5.4 TB/s (268 MB written, 134 read past the L2s): a copy's rate.
template <class T, bool AL, int U>
__global__ void __launch_bounds__(256) embed_kernel(EmbedArgs a, const T* __restrict__ table, const int* __restrict__ ids,
                                                    T* __restrict__ out) {
  constexpr int VE = kVecElems<T>;
  int vec[U], id[U];
  int64_t t[U];
  RowVec<T> v[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    t[u] = item_row(a.nv, vec[u], block_id() * U + u);
    id[u] = t[u] < a.n ? ids[t[u]] : -1;
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = vec[u] * VE;
    if (id[u] >= 0 && id[u] < a.rows) {
      v[u] = load_vec<T, AL>(table + id[u] * a.ld_table + c, a.width - c);
    } else {
#pragma unroll
      for (int q = 0; q < VE; ++q) v[u].e[q] = (T)0.f;
      id[u] = -1;
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (t[u] >= a.n) continue;
    const int c = vec[u] * VE;
    if (id[u] >= 0)
#pragma unroll
      for (int q = 0; q < VE; ++q) v[u].e[q] = (T)(a.scale * to_f32(v[u].e[q]));
    store_vec<T, AL>(out + t[u] * a.ld_out + c, v[u], a.width - c);
  }
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
  int rows, width, nv, seg;   // seg: sorted slots per segment
  int64_t segments;
  int64_t ld_part;         // width in whole vectors
  float scale;
  const int *key, *slot;   // sorted
  float* part;             // [segments][2][ld_part]
  int* last;               // [rows]: of a run over several segments, the last one
  int zero_blocks;         // of the sum's launch, before the sums
};

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
__device__ __forceinline__ void zero_missing(const EmbedGradArgs& a, int block, T* dtable) {
  constexpr int VE = kVecElems<T>;
  const int lane = threadIdx.x & 63;
  const int64_t v0 = ((int64_t)block * 4 + (threadIdx.x >> 6)) * 64;
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

// Sums over the sorted slots: a thread takes 16 bytes of the columns of a segment's rows of
// dout and adds them in their order. A run of equal ids that lies within the segment goes to
// the table; the parts of one that was begun before (0) or goes on behind (1; also where
// it begins at the segment's first slot) go to part, for the join. The launch's first
// blocks look for the rows that do not occur. No thread needs another, so that any width fills the waves. 131,072 rows
// of 1024 bfloat16 into 32,000: 97 us, 272 MB read and 83 written; with 64 slots to a wave that walks
// the columns 211 us, and 33 for the missing rows. Four rows in flight: 125 us for the whole gradient (in a captured
// graph, as at the rules below; its kernels one by one add up to 143), with two 124, eight 132, sixteen 165.
template <class T, bool AL>
__global__ void __launch_bounds__(256) embed_sum_kernel(EmbedGradArgs a, const T* __restrict__ dout, T* __restrict__ dtable) {
  constexpr int VE = kVecElems<T>, U = 4;
  if (block_id() < a.zero_blocks) {
    zero_missing<T, AL>(a, block_id(), dtable);
    return;
  }
  int vec;
  const int64_t seg = item_row(a.nv, vec, block_id() - a.zero_blocks);
  if (seg >= a.segments) return;
  const int64_t r0 = seg * a.seg;
  const int count = (int)min<int64_t>(a.seg, a.n - r0);
  const int *keys = a.key + r0, *slots = a.slot + r0;
  const int before = r0 > 0 ? keys[-1] : -1, after = r0 + count < a.n ? keys[count] : -1;
  const int c = vec * VE, n = a.width - c;
  float acc[VE] = {};
  int key = keys[0];
  bool begun = key == before;
  auto flush = [&](bool goes_on) {
    if (key >= a.rows) return;
    if (begun || goes_on) {
      float* p = a.part + (2 * seg + (begun ? 0 : 1)) * a.ld_part + c;
#pragma unroll
      for (int q = 0; q < VE; q += 4) *reinterpret_cast<f4*>(p + q) = f4{acc[q], acc[q + 1], acc[q + 2], acc[q + 3]};
      if (vec == 0 && !goes_on) a.last[key] = (int)seg;
    } else {
      RowVec<T> o;
#pragma unroll
      for (int q = 0; q < VE; ++q) o.e[q] = (T)(a.scale * acc[q]);
      store_vec<T, AL>(dtable + key * a.ld_table + c, o, n);
    }
  };
  int k[U], sl[U];
  auto look = [&](int r) {   // ids and slots of a batch, requested while the one before is added
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = min(r + u, count - 1);
      k[u] = keys[s], sl[u] = slots[s];
    }
  };
  look(0);
  for (int r = 0; r < count; r += U) {
    RowVec<T> v[U];
    int kr[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      kr[u] = k[u];
      if (kr[u] < a.rows) v[u] = load_vec<T, AL>(dout + sl[u] * a.ld_dout + c, n);
    }
    if (r + U < count) look(r + U);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (r + u >= count) continue;
      if (kr[u] != key) {
        flush(false);
        key = kr[u];
        begun = false;
#pragma unroll
        for (int q = 0; q < VE; ++q) acc[q] = 0.f;
      }
      if (kr[u] < a.rows)
#pragma unroll
        for (int q = 0; q < VE; ++q) acc[q] += to_f32(v[u].e[q]);
    }
  }
  flush(key == after);
}

// Runs that cross segments are joined by the block of the segment they begin in: blocks of JS segments
// and cl lanes of four columns each. The JT / cl groups of lanes take a short run each; a long one's
// parts are shared among all groups, contiguous ones each, and the groups' sums added in order.
constexpr int kShortRun = 8;
template <class T, int JT, int JS>
__global__ void __launch_bounds__(JT) embed_join_kernel(EmbedGradArgs a, int cl, int col_blocks, T* __restrict__ dtable) {
  __shared__ f4 red[JT];
  const int tid = threadIdx.x, lane = tid % cl, group = tid / cl, groups = JT / cl;
  const int64_t s0 = (int64_t)(block_id() / col_blocks) * JS;
  const int col = 4 * (block_id() % col_blocks * cl + lane);
  // lane i of each wave: the run that segment s0 + i begins and others go on with
  const int64_t mine = s0 + (tid & (JS - 1)), end = (mine + 1) * a.seg;
  int key = 0, parts = 0;
  if (mine < a.segments && end < a.n) {
    key = a.key[end - 1];
    const bool begun = mine > 0 && a.key[mine * a.seg] == key && a.key[mine * a.seg - 1] == key;
    if (key < a.rows && a.key[end] == key && !begun) parts = a.last[key] - (int)mine + 1;
  }
  auto sum = [&](int64_t seg, int p0, int p1) {   // parts p0 up to p1 of the run that begins in seg
    f4 s = {0.f, 0.f, 0.f, 0.f};
    if (col < a.ld_part)
      for (int p = p0; p < p1; p += 8) {   // eight loads in flight, added in order
        f4 v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int q = min(p + u, p1 - 1);
          v[u] = *reinterpret_cast<const f4*>(a.part + (2 * (seg + q) + (q == 0)) * a.ld_part + col);
        }
#pragma unroll
        for (int u = 0; u < 8; ++u)
          if (p + u < p1) s += v[u];
      }
    return s;
  };
  auto store = [&](int v, f4 s) {
    const int n = a.width - col;
    if (n > 0) store_n(dtable + v * a.ld_table + col, s * a.scale, min(4, n), false);
  };
  int nth = 0;
  for (int i = 0; i < JS; ++i) {   // short runs
    const int np = __shfl(parts, i), v = __shfl(key, i);
    if (np == 0 || np > kShortRun) continue;
    if (nth++ % groups == group) store(v, sum(s0 + i, 0, np));
  }
  for (int i = 0; i < JS; ++i) {
    const int np = __shfl(parts, i), v = __shfl(key, i);
    if (np <= kShortRun) continue;
    const int per = (np + groups - 1) / groups;
    red[tid] = sum(s0 + i, min(np, group * per), min(np, (group + 1) * per));
    __syncthreads();
    if (group == 0) {
      f4 s = red[lane];
      for (int q = 1; q < groups; ++q) s += red[q * cl + lane];
      store(v, s);
    }
    __syncthreads();
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

// Slots a block of the sort takes at a time: 131,072 ids of 32,000 rows 125 us for the whole gradient, with 1024
// 126 (more blocks' counts to read), with 4096 131 (fewer CUs); 262,144 ids of 2 rows 36.6, 35.5, 39.8.
constexpr int kChunk = 2048;
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
// Slots per segment: enough threads to fill the chip, few enough parts to join. 17,711 ids of 89 rows
// 515 wide: 8 slots 32.6 us, 16 28.1, 32 33.1; 4,000 ids 128 wide: 8 slots 17.3, 16 19.2.
int segment(const mace_embed_desc& d) {
  const int64_t nv = ceil_div(d.width, d.dtype == MACE_TYPE_FP32 ? 4 : 8), least = d.n_ids < 8192 ? 8 : 16;
  return (int)std::max(least, std::min<int64_t>(64, std::max(d.n_ids * nv / (1 << 19), d.n_ids / 8192)));
}

struct BackwardPlan {
  SortPlan sort;
  int seg;
  int64_t segments, ld_part;
  size_t hist, key[2], slot[2], part, last, total;
};
BackwardPlan plan_backward(const mace_embed_desc& d) {
  BackwardPlan p{};
  p.sort = sort_plan(d.n_rows);
  p.seg = segment(d);
  p.segments = ceil_div(d.n_ids, p.seg);
  p.ld_part = ceil_div(d.width, 8) * 8;
  size_t o = 0;
  auto take = [&](size_t bytes) {
    const size_t at = o;
    o += round256(bytes);
    return at;
  };
  p.hist = take(size_t(sort_blocks<kChunk>(d.n_ids)) * (p.sort.buckets() + 1) * sizeof(int));
  for (int i = 0; i < 2; ++i) {
    p.key[i] = take(size_t(d.n_ids) * sizeof(int));
    p.slot[i] = take(size_t(d.n_ids) * sizeof(int));
  }
  p.part = take(size_t(p.segments) * 2 * p.ld_part * sizeof(float));
  p.last = take(size_t(d.n_rows) * sizeof(int));
  p.total = o;
  return p;
}

}  // namespace
}  // namespace mace

using namespace mace;

// Four vectors a thread from 16,384 blocks of one each on: 131,072 rows of 1024 bfloat16 (65,536)
// 81 us against 90, 17,711 of 515 (4,497) 12.0 against 8.5.
constexpr int64_t kManyBlocks = 1 << 14;

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
    const bool al = aligned<T>(d, table, out);
    auto run = [&](auto u) {
      constexpr int U = decltype(u)::value;
      auto f = al ? embed_kernel<T, true, U> : embed_kernel<T, false, U>;
      f<<<grid_of(ceil_div(blocks, U)), 256, 0, (hipStream_t)stream>>>(a, (const T*)table, ids, (T*)out);
    };
    if (blocks >= kManyBlocks) run(Int<4>{});
    else run(Int<1>{});
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
    a.nv = (int)ceil_div(d.width, kVecElems<T>), a.seg = p.seg, a.segments = p.segments, a.scale = (float)d.scale;
    a.ld_part = p.ld_part;
    a.part = reinterpret_cast<float*>(ws + p.part);
    a.last = ints(p.last);
    int cl = 1;
    while (cl < 64 && 4 * cl < d.width) cl *= 2;
    const int64_t col_blocks = ceil_div(d.width, 4 * cl);
    const int64_t zero_blocks = ceil_div(d.n_rows, 256), blocks = zero_blocks + ceil_div(a.segments * a.nv, 256);
    // more lanes to a run where the average one is 128 parts or more to each group of the smaller
    // block: 262,144 ids of 8 rows 797 wide 160 us against 184, 131,072 of 32,000 134 against 125
    const bool long_runs = a.segments / d.n_rows >= 128 * (256 / cl);
    const int64_t join_blocks = ceil_div(a.segments, long_runs ? 16 : 4) * col_blocks;
    if (!fits_grid(blocks) || !fits_grid(join_blocks)) return MACE_EUNSUPPORTED;
    a.zero_blocks = (int)zero_blocks;
    for (int i = 0; i < p.sort.passes && d.n_ids > 0; ++i) {
      const EmbedSlots sl{i ? ints(p.key[(i + 1) & 1]) : ids, i ? ints(p.slot[(i + 1) & 1]) : nullptr, ints(p.key[i & 1]),
                          ints(p.slot[i & 1]), a.rows, i * p.sort.bits, p.sort.buckets() - 1};
      const mace_status e = sort_slots<kChunk>(sl, d.n_ids, p.sort.buckets() - 1, ints(p.hist), nullptr, s);
      if (e != MACE_OK) return e;
    }
    a.key = ints(p.key[(p.sort.passes + 1) & 1]), a.slot = ints(p.slot[(p.sort.passes + 1) & 1]);
    const bool al = aligned<T>(d, dout, dtable);
    auto f = al ? embed_sum_kernel<T, true> : embed_sum_kernel<T, false>;
    f<<<grid_of(blocks), 256, 0, s>>>(a, (const T*)dout, (T*)dtable);
    if ((st = launched()) != MACE_OK || a.segments <= 1) return st;
    if (long_runs) embed_join_kernel<T, 1024, 16><<<grid_of(join_blocks), 1024, 0, s>>>(a, cl, (int)col_blocks, (T*)dtable);
    else embed_join_kernel<T, 256, 4><<<grid_of(join_blocks), 256, 0, s>>>(a, cl, (int)col_blocks, (T*)dtable);
    return launched();
  });
}
