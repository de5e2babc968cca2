// Tiles of dense matrix products on MFMA, shared by the linear and the
// orthogonalisation kernels: operands of FP32, bfloat16, binary16 or pairs of
// binary16 go through LDS as one to three 16-bit planes, and a block multiplies
// them with v_mfma_f32_16x16x32.
#pragma once

#include "mace_internal.h"

namespace mace {

template <int I> struct Int { static constexpr int value = I; };

typedef float f4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef unsigned short us8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));

// A binary16 pair (hi, lo) stored as two planes, `plane` elements apart: 22
// significand bits, for operands whose range is known.
struct HalfPair {};

// Two 8-bit integers, consecutive in k: products of integers go through the tiles as 16-bit
// units of K / 2, a fragment of 8 units being 16 integers.
struct IntPair { unsigned short pair; };
typedef int i4 __attribute__((ext_vector_type(4)));

// Planes an operand is carried as: FP32 as three bfloat16 (x0 + x1 + x2 = x
// exactly, the six partial products down to 2^-18 relative kept, so products
// are as accurate as FP32's), 16-bit types as themselves, pairs as two (three
// partial products kept, the dropped one is 2^-22 relative).
template <class T> struct Planes { static constexpr int n = 1; };
template <> struct Planes<float> { static constexpr int n = 3; };
template <> struct Planes<HalfPair> { static constexpr int n = 2; };

template <class T>
__device__ __forceinline__ f4 mfma32(us8 a, us8 b, f4 c) {
  if constexpr (__is_same(T, IntPair))   // (32-bit integer sums in the accumulator's registers)
    return __builtin_bit_cast(f4, __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i4, a), __builtin_bit_cast(i4, b),
                                                                        __builtin_bit_cast(i4, c), 0, 0, 0));
  else if constexpr (sizeof(T) == 4 || __is_same(T, __bf16))
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
}

// ------------------------------------------------------------------ elements
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__bf16 x) { return (float)x; }
__device__ __forceinline__ float to_f32(_Float16 x) { return (float)x; }

// eight consecutive elements in registers
template <class T> struct Vec8 {
  us8 v;
  __device__ __forceinline__ float get(int i) const { return to_f32(__builtin_bit_cast(T, (unsigned short)v[i])); }
  __device__ __forceinline__ void set(int i, T x) { v[i] = __builtin_bit_cast(unsigned short, x); }
  __device__ __forceinline__ void zero() { v = us8{0, 0, 0, 0, 0, 0, 0, 0}; }
};
template <> struct Vec8<float> {
  f4 v[2];
  __device__ __forceinline__ float get(int i) const { return v[i >> 2][i & 3]; }
  __device__ __forceinline__ void set(int i, float x) { v[i >> 2][i & 3] = x; }
  __device__ __forceinline__ void zero() { v[0] = v[1] = f4{0.f, 0.f, 0.f, 0.f}; }
};

// p[0..7]; AL: p is 16-byte aligned, otherwise aligned to an element only (the
// hardware takes unaligned vector loads, more slowly)
template <class T, bool AL>
__device__ __forceinline__ Vec8<T> load8(const T* p) {
  Vec8<T> r;
  if constexpr (AL) r = *reinterpret_cast<const Vec8<T>*>(p);
  else __builtin_memcpy(&r, p, sizeof(r));
  return r;
}
// p[0..7], zeros from `end` on (AL: there are none)
template <class T, bool AL>
__device__ __forceinline__ Vec8<T> load8_to(const T* p, const T* end) {
  if (AL || p + 8 <= end) return load8<T, AL>(p);
  Vec8<T> r;
  r.zero();
#pragma unroll
  for (int i = 0; i < 7; ++i)
    if (p + i < end) r.set(i, p[i]);
  return r;
}

template <class T>
__device__ __forceinline__ void to_planes(const Vec8<T>& x, us8 (&p)[Planes<T>::n]) {
  if constexpr (sizeof(T) == 4) {
    typedef unsigned u4_ __attribute__((ext_vector_type(4)));
    u4_ w[3];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      unsigned a, b, c;
      split3_pair(f2v{x.get(2 * i), x.get(2 * i + 1)}, a, b, c);
      w[0][i] = a;
      w[1][i] = b;
      w[2][i] = c;
    }
#pragma unroll
    for (int q = 0; q < 3; ++q) p[q] = __builtin_bit_cast(us8, w[q]);
  } else {
    p[0] = x.v;
  }
}

typedef float f8 __attribute__((ext_vector_type(8)));
template <int W> struct Floats { using type = f4; };
template <> struct Floats<8> { using type = f8; };
template <class V> constexpr int width_of = sizeof(V) / 4;

// n <= W consecutive elements from FP32 values, rounded once; vec: n = W and p is
// aligned to W elements. Whole vectors at other places go as unaligned ones.
template <class T, class V>
__device__ __forceinline__ void store_n(T* p, V v, int n, bool vec) {
  constexpr int W = width_of<V>;
  typedef T tw __attribute__((ext_vector_type(W)));
  const tw o = __builtin_convertvector(v, tw);
  if (vec) {
    *reinterpret_cast<tw*>(p) = o;
  } else if (n >= W) {
    __builtin_memcpy(p, &o, sizeof(o));
  } else {
#pragma unroll
    for (int i = 0; i < W - 1; ++i)
      if (i < n) p[i] = o[i];
  }
}
template <int W, class T>
__device__ __forceinline__ auto read_raw(const T* p, int n, bool vec) {   // as the elements are
  typedef T tw __attribute__((ext_vector_type(W)));
  if (vec) return *reinterpret_cast<const tw*>(p);
  tw o = {};
  if (n >= W) {
    __builtin_memcpy(&o, p, sizeof(o));
  } else {
#pragma unroll
    for (int i = 0; i < W - 1; ++i)
      if (i < n) o[i] = p[i];
  }
  return o;
}
template <int W, class T>
__device__ __forceinline__ typename Floats<W>::type read_n(const T* p, int n, bool vec) {
  return __builtin_convertvector(read_raw<W>(p, n, vec), typename Floats<W>::type);
}

// ------------------------------------------------------------------ LDS tiles
// A tile of ROWS operand rows (rows of the first or columns of the second
// factor) by BK products' indices k. KC: k is contiguous in memory, and in LDS
// each row's 16-byte chunks are XORed with the row, so that the 8 rows a
// ds_read_b128 takes per clock cover all banks. Otherwise the rows are
// contiguous: LDS keeps [k][ROWS] and ds_read_b64_tr_b16 transposes (16 lanes
// give 4 x 4 chunks of 4 elements, lane i gets column i of the four rows); the
// 32-byte pairs of a k row are XORed with k, so that its four rows lie apart.
template <int ROWS, int BK, bool KC>
__device__ __forceinline__ int tile_chunk(int row, int k) {   // element offset of the 8-element chunk holding (row, k)
  if constexpr (KC) {
    constexpr int C = BK / 8;
    static_assert(C == 4 || C == 8, "BK is 32 or 64");
    const int s = C == 8 ? row & 7 : (row >> 1) & 3;
    return row * BK + (((k >> 3) ^ s) << 3);
  } else {
    return k * ROWS + (((row >> 3) ^ ((k & 3) << 1)) << 3);
  }
}

// MFMA operand of the 16 rows from row0 and the 32 k from k0: lane l holds
// [row0 + l%16][k0 + 8 (l/16) + 0..7]
template <int ROWS, int BK, bool KC>
__device__ __forceinline__ us8 tile_fragment(const unsigned short* t, int row0, int k0, int lane) {
  const int i = lane & 15, g = lane >> 4;
  if constexpr (KC) {
    return *reinterpret_cast<const us8*>(t + tile_chunk<ROWS, BK, true>(row0 + i, k0 + 8 * g));
  } else {
    typedef __attribute__((address_space(3))) s4 lds_s4;
    const int row = row0 + 4 * (i & 3), k = k0 + 8 * g + (i >> 2);
    const unsigned short* p = t + tile_chunk<ROWS, BK, false>(row, k) + (row & 7);   // (k + 4 has the same k & 3)
    const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)p);
    const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(p + 4 * ROWS));
    typedef short s8_ __attribute__((ext_vector_type(8)));
    const s8_ r = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(us8, r);
  }
}

// Source of a tile in global memory: element (row, k) at base[row * ld + k] (KC)
// or base[k * ld + row]. `rows` >= 1 of the tile's ROWS are in bounds; what is
// read in the places of the others is not used, and every k past the end reads as
// zero. With AL vectors are aligned and whole, and those past the rows repeat the
// last one. Otherwise a vector may run past its row, into the next one or the gap
// before it, but not past `end`, the end of the whole tensor, where it is cut.
// DEPTH sets of registers hold the tiles in flight.
template <class T, int ROWS, int BK, bool KC, bool AL, int NT, int DEPTH = 1>
struct TileSource {
  static constexpr int NV = ROWS * BK / 8 / NT;
  static constexpr int P = Planes<T>::n;
  static_assert(ROWS * BK / 8 % NT == 0, "whole vectors per thread");
  const T* p[NV];
  const T* end;
  Vec8<T> v[DEPTH][NV];
  int64_t step;
  __device__ __forceinline__ static int row_of(int u, int tid) {
    const int f = tid + NT * u;
    return KC ? f / (BK / 8) : 8 * (f % (ROWS / 8));
  }
  __device__ __forceinline__ static int k_of(int u, int tid) {
    const int f = tid + NT * u;
    return KC ? 8 * (f % (BK / 8)) : f / (ROWS / 8);
  }
  __device__ __forceinline__ void init(const T* base, int64_t ld, int rows, int tid, const T* end_ = nullptr) {
    step = KC ? (int64_t)BK : BK * ld;
    end = end_;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int r = row_of(u, tid), k = k_of(u, tid);
      if constexpr (KC) p[u] = base + (int64_t)min(r, rows - 1) * ld + k;
      else if constexpr (AL) p[u] = base + k * ld + min(r, rows - 8);   // (rows is a multiple of 8)
      else p[u] = base + k * ld + r;
    }
  }
  // the tile at the current k into register set D; k_left: products' indices from it to the end
  template <int D = 0>
  __device__ __forceinline__ void load(int k_left, int tid) {
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      if constexpr (AL) {
        if (k_left >= BK) {
          v[D][u] = load8<T, true>(p[u]);
        } else {
          v[D][u].zero();
          if (k_of(u, tid) < k_left) v[D][u] = load8<T, true>(p[u]);
        }
      } else {
        v[D][u] = load8_to<T, false>(p[u], end);
      }
    }
    if (!AL && k_left < BK) {
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        const int n = k_left - k_of(u, tid);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if ((KC ? i : 0) >= n) v[D][u].set(i, T{});
      }
    }
#pragma unroll
    for (int u = 0; u < NV; ++u) p[u] += step;
  }
  template <int D = 0>
  __device__ __forceinline__ void store(unsigned short* t, int tid) const {
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      us8 q[P];
      to_planes<T>(v[D][u], q);
      const int o = tile_chunk<ROWS, BK, KC>(row_of(u, tid), k_of(u, tid));
#pragma unroll
      for (int i = 0; i < P; ++i) *reinterpret_cast<us8*>(t + i * ROWS * BK + o) = q[i];
    }
  }
};

__device__ __forceinline__ uint64_t uniform64(uint64_t v) {
  return ((uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32) |
         (unsigned)__builtin_amdgcn_readfirstlane((int)v);
}

// The same tile of 16-bit elements copied from memory to LDS without passing through
// registers (16-byte aligned rows of whole vectors): a wave's 64 lanes fill 1024
// consecutive bytes, so each lane reads the chunk that the tile's layout wants at its
// place. Whole steps of BK only; the rest of a row goes through TileSource, which
// fills with zeros.
template <int ROWS, int BK, bool KC, int NT>
struct DirectSource {
  static constexpr int NV = ROWS * BK / 8 / NT;
  static_assert(ROWS * BK / 8 % NT == 0, "whole vectors per thread");
  unsigned off[NV];   // bytes from the step's first element (the caller sees to it that they fit)
  uint64_t base, step;
  __device__ __forceinline__ void init(const void* base_, int64_t ld, int rows, int tid) {
    base = uniform64(reinterpret_cast<uint64_t>(base_));
    step = uniform64(2 * (KC ? (uint64_t)BK : BK * ld));
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int f = tid + NT * u;   // the vector at this place of the tile
      if constexpr (KC) {
        constexpr int C = BK / 8;
        const int r = f / C, c = f % C ^ (C == 8 ? r & 7 : (r >> 1) & 3);
        off[u] = 2 * (unsigned)(min(r, rows - 1) * ld + 8 * c);
      } else {
        constexpr int C = ROWS / 8;
        const int k = f / C, c = f % C ^ (k & 3) << 1;
        off[u] = 2 * (unsigned)(k * ld + min(8 * c, rows - 8));
      }
    }
  }
  // Written as asm: the compiler would wait for these copies before any later LDS
  // read, having no way to know that it reads the other buffer. They have no
  // register outputs; tile_gemm_direct waits for them (vmcnt) itself. The s_nop is
  // the wait state between writing M0 and an LDS copy.
  // plane: bytes from the first plane to the one copied
  __device__ __forceinline__ void issue(const unsigned short* t, int64_t plane, int tid) const {
    typedef __attribute__((address_space(3))) const unsigned short las;
    const unsigned at = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(las*)t + (tid & ~63) * 16);
#pragma unroll
    for (int u = 0; u < NV; ++u)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                   :
                   : "s"(at + NT * u * 16), "v"(off[u]), "s"(base + plane)
                   : "memory", "m0");
  }
  __device__ __forceinline__ void next() { base += step; }
};

// The same for pairs of binary16 in two planes, 16-byte aligned rows of whole vectors.
template <int ROWS, int BK, bool KC, int NT>
struct TileSource<HalfPair, ROWS, BK, KC, true, NT> {
  static constexpr int NV = ROWS * BK / 8 / NT;
  static_assert(ROWS * BK / 8 % NT == 0, "whole vectors per thread");
  TileSource<_Float16, ROWS, BK, KC, true, NT> hi;
  int64_t plane;
  us8 lo[NV];
  __device__ __forceinline__ void init(const _Float16* base, int64_t plane_, int64_t ld, int rows, int tid) {
    hi.init(base, ld, rows, tid);
    plane = plane_;
  }
  __device__ __forceinline__ void load(int k_left, int tid) {
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int k = hi.k_of(u, tid);
      lo[u] = us8{0, 0, 0, 0, 0, 0, 0, 0};
      if (k < k_left) lo[u] = *reinterpret_cast<const us8*>(hi.p[u] + plane);
    }
    hi.load(k_left, tid);
  }
  __device__ __forceinline__ void store(unsigned short* t, int tid) const {
    hi.store(t, tid);
#pragma unroll
    for (int u = 0; u < NV; ++u)
      *reinterpret_cast<us8*>(t + ROWS * BK + tile_chunk<ROWS, BK, KC>(hi.row_of(u, tid), hi.k_of(u, tid))) = lo[u];
  }
};

// A block's product: BM rows x BN columns on WM x WN waves, k in steps of BK
// through STAGES LDS buffers. acc[j][i], register r of lane l is the result at
// column 16 j + 4 (l/16) + r and row 16 i + l%16 of the wave's part: four
// consecutive columns of one row per lane.
template <int BM_, int BN_, int WM_, int WN_, int BK_, int STAGES_, bool DIRECT_ = false>
struct TileShape {
  static constexpr bool DIRECT = DIRECT_;   // operands straight to LDS where they are aligned
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, BK = BK_, STAGES = STAGES_;
  static constexpr int DEPTH = STAGES == 1 ? 1 : 2;   // (of tile_gemm)
  static constexpr int NT = 64 * WM * WN;
  static constexpr int TM = BM / WM / 16, TN = BN / WN / 16;   // 16 x 16 tiles per wave
};

// The partial products kept, smallest first: parts of the first and the second factor
template <int P> struct Partial;
template <> struct Partial<1> { static constexpr int n = 1, a[1] = {0}, b[1] = {0}; };
template <> struct Partial<2> { static constexpr int n = 3, a[3] = {1, 0, 0}, b[3] = {0, 1, 0}; };
template <> struct Partial<3> { static constexpr int n = 6, a[6] = {2, 1, 0, 1, 0, 0}, b[6] = {0, 1, 2, 0, 1, 0}; };

// acc[i] += a b[i], the partial products of one i in a row: an MFMA takes the sum
// of the one before it without waiting (with the partial products outside the
// time is the same to 2 %)
template <class T, int P, int N>
__device__ __forceinline__ void products(const us8 (&a)[P], const us8 (&b)[N][P], f4 (&acc)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int q = 0; q < Partial<P>::n; ++q) acc[i] = mfma32<T>(a[Partial<P>::a[q]], b[i][Partial<P>::b[q]], acc[i]);
}

// one BK step out of LDS: rows' planes at tr, columns' at tc
template <class T, class S, bool KCR, bool KCC, int P>
__device__ __forceinline__ void tile_products(const unsigned short* tr, const unsigned short* tc, int m0, int n0, int lane,
                                              f4 (&acc)[S::TN][S::TM]) {
#pragma unroll
  for (int k = 0; k < S::BK; k += 32) {
    us8 b[S::TM][P];
#pragma unroll
    for (int i = 0; i < S::TM; ++i)
#pragma unroll
      for (int q = 0; q < P; ++q) b[i][q] = tile_fragment<S::BM, S::BK, KCR>(tr + q * S::BM * S::BK, m0 + 16 * i, k, lane);
#pragma unroll
    for (int j = 0; j < S::TN; ++j) {
      us8 a[P];
#pragma unroll
      for (int q = 0; q < P; ++q) a[q] = tile_fragment<S::BN, S::BK, KCC>(tc + q * S::BN * S::BK, n0 + 16 * j, k, lane);
      products<T>(a, b, acc[j]);
    }
  }
}

// 16-bit units of LDS of a block
template <class T, class S> constexpr int tile_lds = S::STAGES * Planes<T>::n * (S::BM + S::BN) * S::BK;

// Staged through registers: two LDS buffers and S::DEPTH sets of registers, or one buffer.
template <class T, class S, bool KCR, bool KCC, bool AL>
__device__ __forceinline__ void tile_gemm(TileSource<T, S::BM, S::BK, KCR, AL, S::NT, S::DEPTH>& r,
                                          TileSource<T, S::BN, S::BK, KCC, AL, S::NT, S::DEPTH>& c, int K,
                                          unsigned short* lds, int tid, f4 (&acc)[S::TN][S::TM]) {
  constexpr int P = Planes<T>::n, BUF = P * (S::BM + S::BN) * S::BK, CO = P * S::BM * S::BK;
  const int lane = tid & 63, w = tid >> 6;
  const int m0 = (w / S::WN) * (S::BM / S::WM), n0 = (w % S::WN) * (S::BN / S::WN);
#pragma unroll
  for (int j = 0; j < S::TN; ++j)
#pragma unroll
    for (int i = 0; i < S::TM; ++i) acc[j][i] = f4{0.f, 0.f, 0.f, 0.f};
  if (K <= 0) return;
  r.template load<0>(K, tid);
  c.template load<0>(K, tid);
  if constexpr (S::STAGES == 2) {
    static_assert(S::DEPTH == 2, "two register sets");
    if (K > S::BK) {
      r.template load<1>(K - S::BK, tid);
      c.template load<1>(K - S::BK, tid);
    }
    r.template store<0>(lds, tid);
    c.template store<0>(lds + CO, tid);
    __syncthreads();
    // step at k out of buffer B: request the step after the next, store the next
    auto step = [&](auto b_, int k) {
      constexpr int B = decltype(b_)::value;
      const int left = K - k;
      if (left > 2 * S::BK) {
        r.template load<B>(left - 2 * S::BK, tid);
        c.template load<B>(left - 2 * S::BK, tid);
      }
      tile_products<T, S, KCR, KCC, P>(lds + B * BUF, lds + B * BUF + CO, m0, n0, lane, acc);
      if (left > S::BK) {
        r.template store<1 - B>(lds + (1 - B) * BUF, tid);
        c.template store<1 - B>(lds + (1 - B) * BUF + CO, tid);
      }
      __syncthreads();
    };
    for (int k = 0; k < K; k += 2 * S::BK) {
      step(Int<0>{}, k);
      if (k + S::BK < K) step(Int<1>{}, k + S::BK);
    }
  } else {
    for (int k = 0; k < K; k += S::BK) {
      if (k) __syncthreads();   // the previous step's products have read the tile
      r.template store<0>(lds, tid);
      c.template store<0>(lds + CO, tid);
      __syncthreads();
      if (k + S::BK < K) {
        r.template load<0>(K - k - S::BK, tid);
        c.template load<0>(K - k - S::BK, tid);
      }
      tile_products<T, S, KCR, KCC, P>(lds, lds + CO, m0, n0, lane, acc);
    }
  }
}

// Two column tiles of a row tile as each lane gets them: four consecutive columns
// 4 (l/16) of either. Exchanging the odd 16-lane rows of the one with the even rows
// of the other leaves a lane with eight consecutive columns, 8 (l/32) of tile (l/16)
// % 2: 16-byte accesses of 16-bit results, 64 bytes of a row together in place of
// 32 (81920 x 64 -> 1280 bfloat16: 75 -> 58 us).
__device__ __forceinline__ f8 join_tiles(f4 a, f4 b) {
  f8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    // (not bit casts: of a vector's element they take the vector's first)
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(a[i]), __float_as_uint(b[i]), false, false);
    r[i] = __uint_as_float(s[0]);
    r[4 + i] = __uint_as_float(s[1]);
  }
  return r;
}
// vectors of columns per row tile, and the first column of vector j of lane l
template <int TN, int W> constexpr int lane_vectors = TN * 4 / W;
template <int W>
__device__ __forceinline__ int lane_column(int j, int l) {
  const int g = l >> 4;
  return W == 4 ? 16 * j + 4 * g : 16 * (2 * j + (g & 1)) + 8 * (g >> 1);
}
template <int W, int TN, int TM>
__device__ __forceinline__ typename Floats<W>::type lane_values(const f4 (&acc)[TN][TM], int j, int i) {
  if constexpr (W == 4) return acc[j][i];
  else return join_tiles(acc[2 * j][i], acc[2 * j + 1][i]);
}
// Consecutive columns a lane takes of results of type T
template <class T> constexpr int lane_width = sizeof(T) == 2 ? 8 : 4;

// This lane's results of a block's product, W consecutive columns at a time:
// f(row, column, values, count) (AL: columns come in whole vectors)
template <class S, int W, bool AL, class F>
__device__ __forceinline__ void for_results(const f4 (&acc)[S::TN][S::TM], int rows, int cols, int tid, F f) {
  const int l = tid & 63, w = tid >> 6;
  const int m0 = (w / S::WN) * (S::BM / S::WM) + (l & 15), n0 = (w % S::WN) * (S::BN / S::WN);
#pragma unroll
  for (int i = 0; i < S::TM; ++i) {
    const int m = m0 + 16 * i;
#pragma unroll
    for (int j = 0; j < lane_vectors<S::TN, W>; ++j) {
      const auto v = lane_values<W>(acc, j, i);   // (by every lane: the exchange reads across rows' lanes)
      const int n = n0 + lane_column<W>(j, l);
      if (m < rows && n < cols) f(m, n, v, AL ? W : min(W, cols - n));
    }
  }
}

// One plane of T's elements, or the two planes of pairs.
template <class T> struct Plane0 { using type = T; };
template <> struct Plane0<HalfPair> { using type = _Float16; };

// Waits until at most N copies to LDS are in flight and this wave's LDS reads
// have returned, then meets the block's other waves.
template <int N>
__device__ __forceinline__ void copies_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "i"(N) : "memory");
}

// An operand of tile_gemm_direct: element (row, k) at p[row * ld + k] or
// p[k * ld + row], `rows` in bounds; `plane` elements to a pair's second plane
template <class T>
struct Operand {
  const typename Plane0<T>::type* p;
  int64_t ld;
  int rows;
  int64_t plane;
  const typename Plane0<T>::type* end = nullptr;   // one past the tensor's last element, for unaligned operands
};

// tile_gemm with both operands copied straight to LDS: a ring of STAGES buffers,
// the copies of the next STAGES - 1 steps in flight during a step's products.
template <class T, class S, bool KCR, bool KCC>
__device__ __forceinline__ void tile_gemm_direct(const Operand<T>& ro, const Operand<T>& co, int K, unsigned short* lds,
                                                 int tid, f4 (&acc)[S::TN][S::TM]) {
  static_assert(sizeof(T) != 4, "FP32 is split on its way through registers");
  constexpr int P = Planes<T>::n, CO = P * S::BM * S::BK, BUF = P * (S::BM + S::BN) * S::BK, ST = S::STAGES;
  const int lane = tid & 63, w = tid >> 6;
  const int m0 = (w / S::WN) * (S::BM / S::WM), n0 = (w % S::WN) * (S::BN / S::WN);
#pragma unroll
  for (int j = 0; j < S::TN; ++j)
#pragma unroll
    for (int i = 0; i < S::TM; ++i) acc[j][i] = f4{0.f, 0.f, 0.f, 0.f};
  if (K <= 0) return;
  const int whole = K / S::BK;
  using R = DirectSource<S::BM, S::BK, KCR, S::NT>;
  using C = DirectSource<S::BN, S::BK, KCC, S::NT>;
  constexpr int COPIES = P * (R::NV + C::NV);   // per step and wave
  static_assert((ST - 2) * COPIES < 64, "the counter of copies in flight has six bits");
  R r;
  C c;
  r.init(ro.p, ro.ld, ro.rows, tid);
  c.init(co.p, co.ld, co.rows, tid);
  auto copy = [&](int buffer) {
    unsigned short* t = lds + buffer * BUF;
#pragma unroll
    for (int q = 0; q < P; ++q) {
      r.issue(t + q * S::BM * S::BK, q ? 2 * ro.plane : 0, tid);
      c.issue(t + CO + q * S::BN * S::BK, q ? 2 * co.plane : 0, tid);
    }
    r.next();
    c.next();
  };
  auto multiply = [&](const unsigned short* t) { tile_products<T, S, KCR, KCC, P>(t, t + CO, m0, n0, lane, acc); };
#pragma unroll
  for (int i = 0; i < ST - 1; ++i)
    if (i < whole) copy(i);
  int b = 0;   // buffer of step i
  for (int i = 0; i < whole; ++i) {
    // step i's copies have landed, and every wave has read the buffer of step i - 1
    if (i + ST - 2 < whole) copies_barrier<(ST - 2) * COPIES>();
    else copies_barrier<0>();
    if (i + ST - 1 < whole) copy(b == 0 ? ST - 1 : b - 1);
    multiply(lds + b * BUF);
    b = b + 1 == ST ? 0 : b + 1;
  }
  if (K % S::BK) {
    const int k = whole * S::BK;
    unsigned short* t = lds + b * BUF;   // (read ST steps ago, with a barrier since)
    auto rest = [&](auto source, const Operand<T>& o, bool kc, unsigned short* d) {
      const auto* p = o.p + (kc ? (int64_t)k : k * o.ld);
      if constexpr (P == 2) source.init(p, o.plane, o.ld, o.rows, tid);
      else source.init(p, o.ld, o.rows, tid);
      source.load(K - k, tid);
      source.store(d, tid);
    };
    rest(TileSource<T, S::BM, S::BK, KCR, true, S::NT>{}, ro, KCR, t);
    rest(TileSource<T, S::BN, S::BK, KCC, true, S::NT>{}, co, KCC, t + CO);
    __syncthreads();
    multiply(t);
  }
}

// Blocks of a launch, numbered along x and then along y. An axis takes fewer than 2^32
// threads: a longer one wraps, without an error. grid_of puts at most 2^21 blocks on x
// (of 1024 threads at most) and fills the last row of y: a kernel's blocks past its work
// return.
constexpr int64_t kGridRow = 1 << 21, kGridMost = 1 << 30;
inline bool fits_grid(int64_t blocks) { return blocks <= kGridMost; }
inline dim3 grid_of(int64_t blocks) {
  return dim3((unsigned)(blocks < kGridRow ? blocks : kGridRow), (unsigned)((blocks + kGridRow - 1) / kGridRow));
}
__device__ __forceinline__ int block_id() { return blockIdx.y * gridDim.x + blockIdx.x; }
__device__ __forceinline__ int block_count() { return gridDim.x * gridDim.y; }

// Work items 0..n-1 in the order blocks take them: consecutive block numbers go
// to different XCDs, so each XCD gets a contiguous run of items (neighbours
// share operand rows in its L2).
__device__ __forceinline__ int xcd_order(int b, int n) {
  constexpr int X = 8;
  const int q = n / X, rem = n % X, x = b % X;
  return x * q + min(x, rem) + b / X;
}

// Runs of at most `size` consecutive rows of one group, numbered over all
// groups; then runs of the rows behind the last group (group = n_groups).
// offsets: n_groups + 1 device ints, clamped here to [0, n], a falling pair
// being an empty group; NULL for one group of all rows. Every lane of a wave
// calls it. False: run t does not exist.
struct RowRun {
  int group;
  int64_t row0;
  int rows;
  int first;   // number of the group's first run
};
__device__ __forceinline__ bool find_run(const int* __restrict__ offsets, int n_groups, int64_t n, int size, int t,
                                         RowRun& out) {
  if (!offsets) {
    out.group = 0;
    out.first = 0;
    out.row0 = (int64_t)t * size;
    out.rows = (int)min<int64_t>(size, n - out.row0);
    return out.row0 < n;
  }
  const int lane = threadIdx.x & 63;
  int base = 0;
  for (int g0 = 0; g0 <= n_groups; g0 += 64) {
    const int g = g0 + lane;
    int64_t a = 0, b = 0;
    if (g <= n_groups) {
      a = min<int64_t>(max(offsets[g], 0), n);
      b = g < n_groups ? min<int64_t>(max(offsets[g + 1], 0), n) : n;
    }
    const int runs = b > a ? (int)((b - a + size - 1) / size) : 0;
    int incl = runs;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(incl, d);
      if (lane >= d) incl += o;
    }
    const unsigned long long has = __ballot(base + incl > t);
    if (has) {
      const int src = __ffsll(has) - 1;
      const int first = base + __shfl(incl - runs, src);
      const int64_t a0 = ((int64_t)__shfl((int)(a >> 32), src) << 32) | (unsigned)__shfl((int)a, src);
      const int64_t b0 = ((int64_t)__shfl((int)(b >> 32), src) << 32) | (unsigned)__shfl((int)b, src);
      out.group = g0 + src;
      out.first = first;
      out.row0 = a0 + (int64_t)(t - first) * size;
      out.rows = (int)min<int64_t>(size, b0 - out.row0);
      return true;
    }
    base += __shfl(incl, 63);
  }
  return false;
}

}  // namespace mace
