// The stable counting sort behind routing and the embedding's gradient.
#pragma once

#include <algorithm>

#include "../../include/mace.h"
#include "dense.h"

namespace mace {

constexpr int kSortBuckets = 512;   // besides the one behind them (the counters fit 64 KB of LDS)
constexpr int kSortWaves = 16;
constexpr int kSortThreads = 64 * kSortWaves;
constexpr int kSortChunkMost = 4096;   // slots a block sorts at a time, at most
constexpr int kSortBlocks = 512;   // most blocks: each reads every block's counts

// What is sorted: bucket(s) of slot s, 0 .. E, and place(s, row), which stores that
// slot s comes at `row`.

// slots per bucket of each block's span (consecutive chunks)
template <class Slots>
__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(Slots sl, int64_t slots, int64_t span, int E,
                                                                  int* __restrict__ hist) {
  __shared__ int cnt[kSortBuckets + 1];
  for (int i = threadIdx.x; i <= E; i += kSortThreads) cnt[i] = 0;
  __syncthreads();
  const int64_t s0 = blockIdx.x * span, s1 = min<int64_t>(slots, s0 + span);
  for (int64_t s = s0 + threadIdx.x; s < s1; s += kSortThreads) atomicAdd(&cnt[sl.bucket(s)], 1);
  __syncthreads();
  for (int i = threadIdx.x; i <= E; i += kSortThreads) hist[(size_t)blockIdx.x * (E + 1) + i] = cnt[i];
}

// The stable counting sort into buckets 0 .. E, a span of chunks per block. Each wave owns a contiguous part
// of a chunk; its counters start behind every earlier slot of the same bucket
// (earlier blocks from hist, earlier chunks and waves from their counts), and it ranks 64
// slots at a time by matching buckets across its lanes. Integer counts only: the
// order of the LDS additions does not matter. Up to one chunk the count is its own and
// the sort one launch (96 slots 4 us, bound by the launch); 294,912 slots of 64
// experts 12 to 14 us with the counting launch, 2^26 of 64 experts 470 us.
// offsets [E + 1], or NULL: the first row of each bucket.
template <class Slots, int kSortChunk>
__global__ void __launch_bounds__(kSortThreads)
sort_kernel(Slots sl, int64_t slots, int64_t span, int E, int bits, const int* __restrict__ hist, int* __restrict__ offsets) {
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
      e[i] = s < s1 ? sl.bucket(s) : -1;
      if (e[i] >= 0) atomicAdd(&cnt[w * E1 + e[i]], 1);
    }
  };
  count(s0);
  if (gridDim.x > 1) {
    // threads over (block, bucket): sums of the blocks' counts, eight loads in flight
    const int all = gridDim.x * E1, mine = blockIdx.x * E1;   // (up to this block's counts: of earlier blocks)
    for (int i0 = tid; i0 < all; i0 += 8 * kSortThreads) {
      int h[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int i = i0 + u * kSortThreads;
        h[u] = i < all ? hist[i] : 0;
      }
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (h[u]) {
          const int i = i0 + u * kSortThreads, k = i % E1;
          atomicAdd(&total[k], h[u]);
          if (i < mine) atomicAdd(&next[k], h[u]);
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
        if (offsets && blockIdx.x == 0) offsets[k] = carry + incl - t;
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
        sl.place(s, mine[e[i]] + rank);
      }
      __builtin_amdgcn_wave_barrier();
      if (on && lane == __ffsll(peers) - 1) mine[e[i]] = mine[e[i]] + __popcll(peers);
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// The launches. hist: sort_blocks(slots) * (E + 1) ints where that is more than one block.
template <int kSortChunk = kSortChunkMost>
int64_t sort_chunks(int64_t slots) { return (slots + kSortChunk - 1) / kSortChunk; }
template <int kSortChunk = kSortChunkMost>
int64_t sort_blocks(int64_t slots) {
  const int64_t chunks = sort_chunks<kSortChunk>(slots);
  const int64_t each = std::max<int64_t>(1, (chunks + kSortBlocks - 1) / kSortBlocks);   // chunks per block
  return std::max<int64_t>(1, (chunks + each - 1) / each);
}
template <int kSortChunk = kSortChunkMost, class Slots>
mace_status sort_slots(const Slots& sl, int64_t slots, int E, int* hist, int* offsets, hipStream_t s) {
  const int64_t each = std::max<int64_t>(1, (sort_chunks<kSortChunk>(slots) + kSortBlocks - 1) / kSortBlocks);
  const int64_t blocks = sort_blocks<kSortChunk>(slots), span = each * kSortChunk;
  int bits = 1;
  while ((1 << bits) <= E) ++bits;
  if (blocks > 1) {
    sort_count_kernel<<<(unsigned)blocks, kSortThreads, 0, s>>>(sl, slots, span, E, hist);
    if (hipGetLastError() != hipSuccess) return MACE_EHIP;
  }
  sort_kernel<Slots, kSortChunk><<<(unsigned)blocks, kSortThreads, (kSortWaves + 2) * (E + 1) * sizeof(int), s>>>(sl, slots, span, E, bits, hist,
                                                                                              offsets);
  return hipGetLastError() == hipSuccess ? MACE_OK : MACE_EHIP;
}

}  // namespace mace
