// Rows sorted by expert and back: mace_route_build, mace_route_gather,
// mace_route_combine, mace_route_combine_backward.
#include <algorithm>

#include "../../include/mace.h"
#include "dense.h"

namespace mace {
namespace {

constexpr int kMaxExperts = 512;   // (the sort's counters fit 64 KB of LDS)
constexpr int kSortWaves = 16;
constexpr int kSortThreads = 64 * kSortWaves;
constexpr int kSortChunk = 4096;   // slots a block sorts at a time
constexpr int kSortBlocks = 512;   // most blocks: each reads every block's counts

__device__ __forceinline__ int bucket_of(int e, int E) { return e >= 0 && e < E ? e : E; }

// slots per bucket of each block's span (consecutive chunks)
__global__ void __launch_bounds__(kSortThreads) route_count_kernel(const int* __restrict__ expert, int64_t slots, int64_t span,
                                                                   int E, int* __restrict__ hist) {
  __shared__ int cnt[kMaxExperts + 1];
  for (int i = threadIdx.x; i <= E; i += kSortThreads) cnt[i] = 0;
  __syncthreads();
  const int64_t s0 = blockIdx.x * span, s1 = min<int64_t>(slots, s0 + span);
  for (int64_t s = s0 + threadIdx.x; s < s1; s += kSortThreads) atomicAdd(&cnt[bucket_of(expert[s], E)], 1);
  __syncthreads();
  for (int i = threadIdx.x; i <= E; i += kSortThreads) hist[(size_t)blockIdx.x * (E + 1) + i] = cnt[i];
}

// The stable counting sort, a span of chunks per block. Bucket E holds the dropped
// slots, so the result is a permutation of all slots. Each wave owns a contiguous part
// of a chunk; its counters start behind every earlier slot of the same bucket
// (earlier blocks from hist, earlier chunks and waves from their counts), and it ranks 64
// slots at a time by matching buckets across its lanes. Integer counts only: the
// order of the LDS additions does not matter. Up to one chunk the count is its own and
// the sort one launch (96 slots 3.5 us, bound by the launch); 294,912 slots of 64
// experts 14 us with the counting launch, 2^26 of 64 experts 470 us.
__global__ void __launch_bounds__(kSortThreads)
route_sort_kernel(const int* __restrict__ expert, int64_t slots, int64_t span, int E, int bits, const int* __restrict__ hist,
                  int* __restrict__ row_of_slot, int* __restrict__ slot_of_row, int* __restrict__ offsets) {
  extern __shared__ int sm[];
  const int E1 = E + 1, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  int* cnt = sm;                       // [waves][E1]
  int* next = cnt + kSortWaves * E1;   // [E1] slots of the bucket in earlier blocks, then its next row
  int* total = next + E1;              // [E1] slots of the bucket in all blocks, then its first row
  for (int i = tid; i < (kSortWaves + 2) * E1; i += kSortThreads) sm[i] = 0;
  __syncthreads();
  const int64_t s0 = blockIdx.x * span, s1 = min<int64_t>(slots, s0 + span);
  constexpr int per = kSortChunk / kSortWaves;
  int e[per / 64];
  auto count = [&](int64_t c0) {   // the chunk's buckets, counted per wave
#pragma unroll
    for (int i = 0; i < per / 64; ++i) {
      const int64_t s = c0 + w * per + 64 * i + lane;
      e[i] = s < s1 ? bucket_of(expert[s], E) : -1;
      if (e[i] >= 0) atomicAdd(&cnt[w * E1 + e[i]], 1);
    }
  };
  count(s0);
  if (gridDim.x > 1) {
    // groups of threads over (block, bucket): partial sums of the blocks' counts
    for (int i = tid; i < (int)gridDim.x * E1; i += kSortThreads) {
      const int b = i / E1, k = i - b * E1, h = hist[i];
      if (h) {
        atomicAdd(&total[k], h);
        if (b < (int)blockIdx.x) atomicAdd(&next[k], h);
      }
    }
    __syncthreads();
  } else {
    __syncthreads();
    for (int k = tid; k < E1; k += kSortThreads) {
      int t = 0;
      for (int v = 0; v < kSortWaves; ++v) t += cnt[v * E1 + k];
      total[k] = t;
    }
    __syncthreads();
  }
  if (w == 0) {   // first row of each bucket
    int carry = 0;
    for (int k0 = 0; k0 < E1; k0 += 64) {
      const int k = k0 + lane;
      const int t = k < E1 ? total[k] : 0;
      int incl = t;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(incl, d);
        if (lane >= d) incl += o;
      }
      if (k < E1) {
        total[k] = carry + incl - t;
        if (blockIdx.x == 0) offsets[k] = carry + incl - t;   // (k = E: the rows kept)
      }
      carry += __shfl(incl, 63);
    }
  }
  __syncthreads();
  for (int k = tid; k < E1; k += kSortThreads) next[k] += total[k];   // (a thread keeps its buckets from here on)
  volatile int* mine = cnt + w * E1;
  for (int64_t c0 = s0; c0 < s1; c0 += kSortChunk) {
    if (c0 > s0) {
      __syncthreads();   // every wave has ranked the chunk before
      for (int i = tid; i < kSortWaves * E1; i += kSortThreads) cnt[i] = 0;
      __syncthreads();
      count(c0);
      __syncthreads();
    }
    for (int k = tid; k < E1; k += kSortThreads) {   // counters: the wave's first row per bucket
      int at = next[k];
      for (int v = 0; v < kSortWaves; ++v) {
        const int c = cnt[v * E1 + k];
        cnt[v * E1 + k] = at;
        at += c;
      }
      next[k] = at;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < per / 64; ++i) {
      const int64_t s = c0 + w * per + 64 * i + lane;
      const bool on = e[i] >= 0;
      unsigned long long peers = __ballot(on);
      for (int b = 0; b < bits; ++b) {
        const unsigned long long m = __ballot(on && (e[i] >> b & 1));
        peers &= (e[i] >> b & 1) ? m : ~m;
      }
      if (on) {
        const int rank = __popcll(peers & ((1ull << lane) - 1));
        const int row = mine[e[i]] + rank;
        row_of_slot[s] = row;
        slot_of_row[row] = (int)s;
      }
      __builtin_amdgcn_wave_barrier();
      if (on && lane == __ffsll(peers) - 1) mine[e[i]] = mine[e[i]] + __popcll(peers);
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// ------------------------------------------------------------------ rows
// 16 bytes of a row: VE elements, at column VE v; the last vector of a row may
// be short. AL: rows and columns keep every vector 16-byte aligned and whole.
template <class T> constexpr int kVecElems = 16 / sizeof(T);
template <class T>
struct RowVec {
  T e[kVecElems<T>];
};
template <class T, bool AL>
__device__ __forceinline__ RowVec<T> load_vec(const T* p, int n) {
  RowVec<T> r;
  if (AL || n >= kVecElems<T>) {
    if constexpr (AL) *reinterpret_cast<uint4*>(&r) = *reinterpret_cast<const uint4*>(p);
    else __builtin_memcpy(&r, p, 16);
  } else {
#pragma unroll
    for (int i = 0; i < kVecElems<T>; ++i) r.e[i] = i < n ? p[i] : (T)0.f;
  }
  return r;
}
template <class T, bool AL>
__device__ __forceinline__ void store_vec(T* p, const RowVec<T>& r, int n) {
  if (AL || n >= kVecElems<T>) {
    if constexpr (AL) *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(&r);
    else __builtin_memcpy(p, &r, 16);
  } else {
#pragma unroll
    for (int i = 0; i < kVecElems<T>; ++i)
      if (i < n) p[i] = r.e[i];
  }
}

struct RouteArgs {
  int64_t n, ld_tokens, ld_rows;
  unsigned last;   // n k - 1: a row index read from memory is held to it
  int k, E, width, nv;
  const int *row_of_slot, *offsets;
};

// Item block_id() * 256 + threadIdx.x as (row, vector) of rows of nv vectors, with
// one division of 64 bits per block.
__device__ __forceinline__ int64_t item_row(int nv, int& vec) {
  const uint64_t i0 = (uint64_t)block_id() * 256;
  const uint64_t q0 = i0 >> 32 ? i0 / (unsigned)nv : (unsigned)i0 / (unsigned)nv;
  const unsigned j = (unsigned)(i0 - q0 * (unsigned)nv) + threadIdx.x, q = j / (unsigned)nv;
  vec = (int)(j - q * (unsigned)nv);
  return (int64_t)(q0 + q);
}

// rows[r] = x[slot_of_row[r] / k], zeros from the first dropped row on. In the rows'
// order: they are written one after the other, and a token is read k times, each time
// past the L2s (36,864 tokens to 8 experts, 1024 bfloat16 wide: 183 us, 606 MB read and
// as many written, 6.5 TB/s; in the tokens' order, read once and written k times, 199).
template <class T, bool AL>
__global__ void __launch_bounds__(256) route_gather_kernel(RouteArgs a, const int* __restrict__ slot_of_row,
                                                           const T* __restrict__ x, T* __restrict__ rows) {
  int vec;
  const int64_t r = item_row(a.nv, vec);
  if (r > a.last) return;
  const int c = vec * kVecElems<T>, n = a.width - c;
  RowVec<T> v;
  if (r < a.offsets[a.E]) {
    const int64_t t = min((unsigned)slot_of_row[r], a.last) / (unsigned)a.k;
    v = load_vec<T, AL>(x + t * a.ld_tokens + c, n);
  } else {
#pragma unroll
    for (int q = 0; q < kVecElems<T>; ++q) v.e[q] = (T)0.f;
  }
  store_vec<T, AL>(rows + r * a.ld_rows + c, v, n);
}

// out[t] = sum_s weight[t, s] rows[row_of_slot[t, s]] over the kept slots, in
// the slots' order, in FP32, rounded once. Dropped slots' rows are not used,
// whatever they hold. One thread per 16 bytes of a token. 36,864 x 8 rows of 1024
// bfloat16: 160 us, 4.2 TB/s where a large copy reaches 5.2; nearly all of it are reads.
template <class T, bool AL, int U>
__global__ void __launch_bounds__(256)
route_combine_kernel(RouteArgs a, const T* __restrict__ rows, const float* __restrict__ weights, T* __restrict__ out) {
  constexpr int VE = kVecElems<T>;
  int vec;
  const int64_t t = item_row(a.nv, vec);
  if (t >= a.n) return;
  const int c = vec * VE, n = a.width - c;
  const int live = a.offsets[a.E];
  float acc[VE] = {};
  for (int s0 = 0; s0 < a.k; s0 += U) {
    RowVec<T> v[U];
    float w[U];
    bool on[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {   // U rows' loads in flight
      const int64_t slot = t * a.k + min(s0 + u, a.k - 1);
      const int r = min((unsigned)a.row_of_slot[slot], a.last);
      on[u] = s0 + u < a.k && r < live;
      w[u] = weights ? weights[slot] : 1.f;
      if (on[u]) v[u] = load_vec<T, AL>(rows + (int64_t)r * a.ld_rows + c, n);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (on[u])
#pragma unroll
        for (int q = 0; q < VE; ++q) acc[q] = __builtin_fmaf(w[u], to_f32(v[u].e[q]), acc[q]);
  }
  RowVec<T> o;
#pragma unroll
  for (int q = 0; q < VE; ++q) o.e[q] = (T)acc[q];
  store_vec<T, AL>(out + t * a.ld_tokens + c, o, n);
}

// drows[row] = weight dout[t] and dweights[t, s] = <rows[row], dout[t]>, zeros
// for dropped slots. LG lanes (a power of two) per token, U slots at a time, dout read
// once for U rows. 36,864 x 8 rows of 1024 bfloat16: 244 us, 5.6 TB/s of memory
// traffic (rows and dout read, gradients written): a large copy's rate.
template <class T, bool AL, int U>
__global__ void __launch_bounds__(256)
route_combine_bwd_kernel(RouteArgs a, int lg, const T* __restrict__ dout, const T* __restrict__ rows,
                         const float* __restrict__ weights, T* __restrict__ drows, float* __restrict__ dweights) {
  constexpr int VE = kVecElems<T>;
  const int lane = threadIdx.x & (lg - 1);
  const int64_t t = ((int64_t)block_id() * 256 + threadIdx.x) / lg;
  if (t >= a.n) return;   // (whole groups of lanes)
  const int live = a.offsets[a.E];
  for (int s0 = 0; s0 < a.k; s0 += U) {
    float dot[U] = {};
    int r[U];
    float w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t slot = t * a.k + min(s0 + u, a.k - 1);
      r[u] = min((unsigned)a.row_of_slot[slot], a.last);
      w[u] = weights ? weights[slot] : 1.f;
    }
    for (int v = lane; v < a.nv; v += lg) {
      const int c = v * VE, n = a.width - c;
      const RowVec<T> g = load_vec<T, AL>(dout + t * a.ld_tokens + c, n);
      RowVec<T> y[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (s0 + u < a.k && r[u] < live && dweights) y[u] = load_vec<T, AL>(rows + (int64_t)r[u] * a.ld_rows + c, n);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (s0 + u >= a.k) continue;
        const bool on = r[u] < live;
        if (on && dweights)
#pragma unroll
          for (int q = 0; q < VE; ++q) dot[u] = __builtin_fmaf(to_f32(y[u].e[q]), to_f32(g.e[q]), dot[u]);
        if (drows) {
          RowVec<T> o;
#pragma unroll
          for (int q = 0; q < VE; ++q) o.e[q] = on ? (T)(w[u] * to_f32(g.e[q])) : (T)0.f;
          store_vec<T, AL>(drows + (int64_t)r[u] * a.ld_rows + c, o, n);
        }
      }
    }
    if (dweights)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        for (int d = lg >> 1; d; d >>= 1) dot[u] += __shfl_xor(dot[u], d);
        if (lane == 0 && s0 + u < a.k) dweights[t * a.k + s0 + u] = dot[u];
      }
  }
}

// ------------------------------------------------------------------ host
mace_status check(const mace_route_desc* d) {
  if (!d || d->n_tokens < 0 || d->top_k < 1 || d->n_experts < 1 || d->width < 1) return MACE_EINVAL;
  if (d->dtype < MACE_TYPE_FP32 || d->dtype > MACE_TYPE_FP16) return MACE_EINVAL;
  if (d->ld_tokens < d->width || d->ld_rows < d->width) return MACE_EINVAL;
  if (d->n_experts > kMaxExperts || d->width > (1 << 20) || d->top_k > (1 << 20) || d->n_tokens > (1 << 30) ||
      d->n_tokens * d->top_k > (1 << 30))
    return MACE_EUNSUPPORTED;
  return MACE_OK;
}
int64_t chunks(const mace_route_desc& d) { return (d.n_tokens * d.top_k + kSortChunk - 1) / kSortChunk; }
mace_status launched() { return hipGetLastError() == hipSuccess ? MACE_OK : MACE_EHIP; }
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

template <class T>
RouteArgs args_of(const mace_route_desc& d, const int* row_of_slot, const int* offsets) {
  const int ve = kVecElems<T>;
  return {d.n_tokens, d.ld_tokens, d.ld_rows, (unsigned)(d.n_tokens * d.top_k - 1), d.top_k, d.n_experts, d.width, (d.width + ve - 1) / ve, row_of_slot, offsets};
}
template <class T>
bool aligned(const mace_route_desc& d, const void* a, const void* b, const void* c = nullptr) {
  const int ve = kVecElems<T>;
  return aligned16(a) && aligned16(b) && aligned16(c) && d.width % ve == 0 && d.ld_tokens % ve == 0 && d.ld_rows % ve == 0;
}

// Slots a thread has in flight: more than four cost combine more waves than they gain
// (eight slots: 176 us with eight in flight, 160 with four).
template <class F>
mace_status by_slots(int k, F f) {
  if (k == 1) return f(Int<1>{});
  return k == 2 ? f(Int<2>{}) : f(Int<4>{});
}
template <class F>
mace_status by_type(int dtype, F f) {
  if (dtype == MACE_TYPE_FP32) return f(0.f);
  if (dtype == MACE_TYPE_BF16) return f((__bf16)0.f);
  return f((_Float16)0.f);
}

}  // namespace
}  // namespace mace

using namespace mace;

extern "C" size_t mace_route_workspace_bytes(const mace_route_desc* desc) {
  if (check(desc) != MACE_OK) return 0;
  return 256 + (size_t)std::min<int64_t>(chunks(*desc), kSortBlocks) * (desc->n_experts + 1) * sizeof(int);
}

extern "C" mace_status mace_route_build(const mace_route_desc* desc, const int32_t* expert, int32_t* row_of_slot,
                                        int32_t* slot_of_row, int32_t* offsets, void* workspace, size_t workspace_bytes,
                                        void* stream) {
  mace_status st = check(desc);
  if (st != MACE_OK) return st;
  const int64_t slots = desc->n_tokens * desc->top_k;
  if (!offsets || (slots > 0 && (!expert || !row_of_slot || !slot_of_row))) return MACE_EINVAL;
  const int E = desc->n_experts;
  const int64_t each = std::max<int64_t>(1, (chunks(*desc) + kSortBlocks - 1) / kSortBlocks);   // chunks per block
  const int64_t blocks = std::max<int64_t>(1, (chunks(*desc) + each - 1) / each), span = each * kSortChunk;
  int* hist = reinterpret_cast<int*>((reinterpret_cast<uintptr_t>(workspace) + 3) & ~uintptr_t(3));
  if (blocks > 1) {
    if (!workspace) return MACE_EINVAL;
    if (workspace_bytes < mace_route_workspace_bytes(desc)) return MACE_ENOSPACE;
  }
  hipStream_t s = (hipStream_t)stream;
  int bits = 1;
  while ((1 << bits) <= E) ++bits;
  if (blocks > 1) {
    route_count_kernel<<<(unsigned)blocks, kSortThreads, 0, s>>>(expert, slots, span, E, hist);
    if ((st = launched()) != MACE_OK) return st;
  }
  route_sort_kernel<<<(unsigned)blocks, kSortThreads, (kSortWaves + 2) * (E + 1) * sizeof(int), s>>>(
      expert, slots, span, E, bits, hist, row_of_slot, slot_of_row, offsets);
  return launched();
}

extern "C" mace_status mace_route_gather(const mace_route_desc* desc, const void* tokens, const int32_t* slot_of_row,
                                         const int32_t* offsets, void* rows, void* stream) {
  const mace_status st = check(desc);
  if (st != MACE_OK) return st;
  if (desc->n_tokens == 0) return MACE_OK;
  if (!tokens || !slot_of_row || !offsets || !rows) return MACE_EINVAL;
  return by_type(desc->dtype, [&](auto zero) {
    using T = decltype(zero);
    const RouteArgs a = args_of<T>(*desc, nullptr, offsets);
    const int64_t blocks = (a.n * a.k * a.nv + 255) / 256;
    if (!fits_grid(blocks)) return MACE_EUNSUPPORTED;
    auto f = aligned<T>(*desc, tokens, rows) ? route_gather_kernel<T, true> : route_gather_kernel<T, false>;
    f<<<grid_of(blocks), 256, 0, (hipStream_t)stream>>>(a, slot_of_row, (const T*)tokens, (T*)rows);
    return launched();
  });
}

extern "C" mace_status mace_route_combine(const mace_route_desc* desc, const void* rows, const float* weights,
                                          const int32_t* row_of_slot, const int32_t* offsets, void* out, void* stream) {
  const mace_status st = check(desc);
  if (st != MACE_OK) return st;
  if (desc->n_tokens == 0) return MACE_OK;
  if (!rows || !row_of_slot || !offsets || !out) return MACE_EINVAL;
  return by_type(desc->dtype, [&](auto zero) {
    using T = decltype(zero);
    const RouteArgs a = args_of<T>(*desc, row_of_slot, offsets);
    const int64_t blocks = (a.n * a.nv + 255) / 256;
    if (!fits_grid(blocks)) return MACE_EUNSUPPORTED;
    return by_slots(a.k, [&](auto u) {
      constexpr int U = decltype(u)::value;
      auto f = aligned<T>(*desc, rows, out) ? route_combine_kernel<T, true, U> : route_combine_kernel<T, false, U>;
      f<<<grid_of(blocks), 256, 0, (hipStream_t)stream>>>(a, (const T*)rows, weights, (T*)out);
      return launched();
    });
  });
}

extern "C" mace_status mace_route_combine_backward(const mace_route_desc* desc, const void* dout, const void* rows,
                                                   const float* weights, const int32_t* row_of_slot,
                                                   const int32_t* offsets, void* drows, float* dweights, void* stream) {
  const mace_status st = check(desc);
  if (st != MACE_OK) return st;
  if (desc->n_tokens == 0) return MACE_OK;
  if (!dout || !row_of_slot || !offsets || (dweights && !rows)) return MACE_EINVAL;
  return by_type(desc->dtype, [&](auto zero) {
    using T = decltype(zero);
    const RouteArgs a = args_of<T>(*desc, row_of_slot, offsets);
    int lg = 1;
    while (lg < 64 && lg < a.nv) lg *= 2;
    const int64_t blocks = (a.n * lg + 255) / 256;
    if (!fits_grid(blocks)) return MACE_EUNSUPPORTED;
    return by_slots(a.k, [&](auto u) {
      constexpr int U = decltype(u)::value;
      auto f = aligned<T>(*desc, dout, rows, drows) ? route_combine_bwd_kernel<T, true, U> : route_combine_bwd_kernel<T, false, U>;
      f<<<grid_of(blocks), 256, 0, (hipStream_t)stream>>>(a, lg, (const T*)dout, (const T*)rows, weights, (T*)drows, dweights);
      return launched();
    });
  });
}
