// Newton-Schulz orthogonalisation: mace_orthogonalise.
//
// Every matrix is kept as x [m][n] with m <= n (a tall one transposed), as pairs
// of binary16 scaled by kScaleX: the iteration's operands are bounded (singular
// values of x below 3.4, checked for the coefficients on the host), so a pair's
// 22 significand bits are as accurate as FP32 here at three MFMA products
// in place of six. Per step: A = x x^T and B = b A + c A A, both symmetric (one
// half computed, the other mirrored), x <- a x + B x.
//
// With few rows (kGramMax, kGramMaxLong) the iteration runs on A alone, in FP64: every x is a
// polynomial of A_0 = x_0 x_0^T times x_0, so A <- P A P and Q <- P Q with
// P = a + b A + c A A, and the result is Q x_0: two passes over the data instead of
// two per step. FP64 because A holds the squares of the singular values and a
// small one's error grows with the square of the value: in 2^-24 arithmetic a
// singular value of 0.003 would be off by a percent, in FP64 by 1e-11.
// A zero singular value's place in A holds a rounding error, 2^-53, of either sign;
// a step multiplies it by up to a^2, and a negative one has no plateau that would
// stop it. Steps that could take it past 2^-13 (kGramGrowth; 10 of the default ones,
// 33 of (1.5, -0.5, 0)) therefore go to the kernels that iterate x, where x x^T is new
// in every step.
#include <algorithm>
#include <cmath>

#include "../../include/mace.h"
#include "dense.h"

namespace mace {
namespace {

// Scales of the operands where the largest singular value is at least one half and b A +
// c A A at least one; where steps leave less, x, A and B are scaled up by powers of two
// (range_of), so that a pair's smallest digits are never what counts. A's scale is the
// square of x's over kScaleX in all cases.
constexpr float kScaleX = 4096.f, kScaleA = 4096.f, kScaleB = 256.f;
constexpr double kMaxSigma = 3.4, kMaxB = 200.0;   // 3.4^2 kScaleA and 200 kScaleB fit binary16
constexpr int kMaxSteps = 64;
// A step on scaled operands, B <- b A + c (A A) and x <- a x + u (B x)
struct ScaledSteps {
  float a[kMaxSteps], u[kMaxSteps], b[kMaxSteps], c[kMaxSteps];
  int n;
};

// one matrix's planes: hi [rows][ld], then lo
struct PairMat {
  _Float16* p;
  int64_t stride, plane;   // between matrices, between planes
  int ld;
};

typedef _Float16 h4 __attribute__((ext_vector_type(4)));
template <int W = 4>
__device__ __forceinline__ typename Floats<W>::type read_pair(const _Float16* p, int64_t plane) {
  return read_n<W>(p, W, true) + read_n<W>(p + plane, W, true);
}
template <class V, class H>
__device__ __forceinline__ void split_pair(V v, H& hi, H& lo) {
  hi = __builtin_convertvector(v, H);
  lo = __builtin_convertvector(v - __builtin_convertvector(hi, V), H);
}

// ------------------------------------------------------------------ norm and packing
constexpr int kNormBlocks = 256;   // most partial sums per matrix

template <class T>
__global__ void __launch_bounds__(256) ns_norm_kernel(const T* __restrict__ g, int64_t stride, int64_t ld, int rows,
                                                      int cols, double* __restrict__ part) {
  __shared__ double red[4];
  const T* m = g + (int64_t)blockIdx.y * stride;
  double s = 0.0;
  for (int r = blockIdx.x * 4 + (threadIdx.x >> 6); r < rows; r += 4 * gridDim.x)   // a row per wave
    for (int c = threadIdx.x & 63; c < cols; c += 64) {
      const double v = to_f32(m[r * ld + c]);
      s += v * v;
    }
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = red[0] + red[1] + red[2] + red[3];
}

// 1 / (|g| + eps) from the partial sums, by every wave alike
__device__ __forceinline__ double ns_scale(const double* part, int n, double eps) {
  double s = 0.0;
  for (int i = threadIdx.x & 63; i < n; i += 64) s += part[i];
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
  return 1.0 / (sqrt(s) + eps);
}

// x = g / (|g| + eps) as pairs, a tall g transposed; zeros in the padding of x, A and B.
// One 64 x 64 tile of x per block.
template <class T>
__global__ void __launch_bounds__(256)
ns_pack_kernel(const T* __restrict__ g, int64_t stride, int64_t ld, int m, int n, bool tall,
               const double* __restrict__ part, int parts, double eps, PairMat x, PairMat A, PairMat B) {
  __shared__ float t[64][65];
  const int b = blockIdx.z, i0 = blockIdx.y * 64, j0 = blockIdx.x * 64, tid = threadIdx.x;
  const T* src = g + (int64_t)b * stride;
  const double inv = ns_scale(part + (int64_t)b * parts, parts, eps) * kScaleX;
  for (int e = tid; e < 64 * 64; e += 256) {
    const int r = e >> 6, c = e & 63;   // c along g's contiguous axis
    const int i = tall ? c : r, j = tall ? r : c;
    float v = 0.f;
    if (i0 + i < m && j0 + j < n)
      v = (float)(to_f32(tall ? src[(int64_t)(j0 + j) * ld + i0 + i] : src[(int64_t)(i0 + i) * ld + j0 + j]) * inv);
    t[i][j] = v;
  }
  __syncthreads();
  _Float16* xp = x.p + b * x.stride;
  for (int e = tid; e < 64 * 16; e += 256) {
    const int i = e >> 4, j = 4 * (e & 15);
    if (i0 + i >= m || j0 + j >= x.ld) continue;
    h4 hi, lo;
    split_pair(f4{t[i][j], t[i][j + 1], t[i][j + 2], t[i][j + 3]}, hi, lo);
    _Float16* o = xp + (int64_t)(i0 + i) * x.ld + j0 + j;
    *reinterpret_cast<h4*>(o) = hi;
    *reinterpret_cast<h4*>(o + x.plane) = lo;
  }
  if (blockIdx.x == 0)
    for (int e = tid; e < 64 * (A.ld - m); e += 256) {
      const int i = i0 + e / (A.ld - m), j = m + e % (A.ld - m);
      if (i >= m) continue;
      for (int q = 0; q < 2; ++q) {
        A.p[b * A.stride + q * A.plane + (int64_t)i * A.ld + j] = (_Float16)0.f;
        B.p[b * B.stride + q * B.plane + (int64_t)i * B.ld + j] = (_Float16)0.f;
      }
    }
}

// no steps: out = g / (|g| + eps)
template <class T>
__global__ void __launch_bounds__(256)
ns_scale_kernel(const T* __restrict__ g, int64_t stride, int64_t ld, int rows, int cols, const double* __restrict__ part,
                int parts, double eps, T* __restrict__ out, int64_t ostride, int64_t old) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const double inv = ns_scale(part + (int64_t)blockIdx.y * parts, parts, eps);
  if (i >= (int64_t)rows * cols) return;
  const int64_t r = i / cols, c = i % cols;
  out[blockIdx.y * ostride + r * old + c] = (T)(float)(to_f32(g[blockIdx.y * stride + r * ld + c]) * inv);
}

// ------------------------------------------------------------------ few rows
// FP64 up to 32 rows, and up to 64 of matrices too long for LDS
constexpr int kGramMax = 32, kGramMaxLong = 64, kGramChunk = 256;
constexpr double kGramGrowth = 0x1p40;
constexpr int kFitMax = 128;   // longest side of a matrix iterated in LDS

// element (i, j) of x's layout in g
template <class T>
__device__ __forceinline__ float element(const T* g, int64_t ld, bool tall, int i, int j) {
  return to_f32(tall ? g[(int64_t)j * ld + i] : g[(int64_t)i * ld + j]);
}

// Squares of R = 16, 32 or 64 rows, padded with zeros, on FP64 MFMA
// (v_mfma_f64_16x16x4: lane l holds A[l%16][l/16] and B[l/16][l%16], register r of the
// result is D[l/16 + 4 r][l%16]), a 16 x 16 tile per wave; R = 16 leaves three of four
// waves idle.
typedef double d4 __attribute__((ext_vector_type(4)));
template <int R> constexpr int kThreads64 = R == 64 ? 1024 : 256;
template <int R> struct Square { double v[R][R + 1]; };
template <int R> struct Columns { float v[R][kGramChunk + 2]; };   // (a column of the four k groups per bank)

template <int R, class F>
__device__ __forceinline__ void each64(int tid, const d4& acc, F f) {   // f(row, column, value)
  const int l = tid & 63, w = tid >> 6;
  if (w >= (R / 16) * (R / 16)) return;
#pragma unroll
  for (int q = 0; q < 4; ++q) f(16 * (w / (R / 16)) + (l >> 4) + 4 * q, 16 * (w % (R / 16)) + (l & 15), acc[q]);
}
// this wave's tile of A B over K, a(row, k) and b(k, column)
template <int R, class FA, class FB>
__device__ __forceinline__ d4 multiply64(int tid, int K, FA a, FB b) {
  const int l = tid & 63, w = tid >> 6, i = l & 15, g = l >> 4;
  d4 acc = {0.0, 0.0, 0.0, 0.0};
  if (w >= (R / 16) * (R / 16)) return acc;
  const int r = 16 * (w / (R / 16)) + i, c = 16 * (w % (R / 16)) + i;
#pragma unroll 8
  for (int k = 0; k < K; k += 4) acc = __builtin_amdgcn_mfma_f64_16x16x4f64(a(r, k + g), b(k + g, c), acc, 0, 0, 0);
  return acc;
}

// columns j0 .. j0 + kGramChunk of x's layout, zeros outside it; all loads in flight at once
template <int R, class T>
__device__ __forceinline__ void load_columns(Columns<R>& t, const T* src, int64_t ld, int m, int n, int j0, bool tall, int tid) {
  constexpr int NT = kThreads64<R>, U = R * kGramChunk / NT;
  const int w = min(kGramChunk, n - j0);
  auto place = [&](int u, int& i, int& j) {   // lanes along g's contiguous axis
    const int e = tid + NT * u;
    i = tall ? e % R : e / kGramChunk;
    j = tall ? e / R : e % kGramChunk;
  };
  T v[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    int i, j;
    place(u, i, j);
    i = min(i, m - 1);
    j = j0 + min(j, w - 1);
    v[u] = tall ? src[(int64_t)j * ld + i] : src[(int64_t)i * ld + j];
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    int i, j;
    place(u, i, j);
    t.v[i][j] = i < m && j < w ? to_f32(v[u]) : 0.f;
  }
}
// A = t t^T of the chunk's columns
template <int R>
__device__ __forceinline__ d4 gram64(const Columns<R>& t, int w, int tid) {
  return multiply64<R>(tid, (w + 3) & ~3, [&](int r, int k) { return (double)t.v[r][k]; },
                       [&](int k, int c) { return (double)t.v[c][k]; });
}
// the iteration on A = g g^T: Q <- Q / (|g| + eps), |g|^2 being the trace of A
struct NsSteps {
  double c[kMaxSteps][3];
  int n;
};
template <int R>
__device__ __forceinline__ void iterate64(Square<R>& A, Square<R>& P, Square<R>& Q, Square<R>& T, double& s_inv, double eps,
                                          const NsSteps& steps, int tid) {
  if (tid < 64) {
    double tr = tid < R ? A.v[tid][tid] : 0.0;
    for (int d = 32; d; d >>= 1) tr += __shfl_xor(tr, d);
    if (tid == 0) s_inv = 1.0 / (sqrt(tr) + eps);
  }
  __syncthreads();
  const double inv = s_inv;
  for (int e = tid; e < R * R; e += kThreads64<R>) {
    A.v[e / R][e % R] *= inv * inv;
    Q.v[e / R][e % R] = e / R == e % R ? 1.0 : 0.0;
  }
  __syncthreads();
  auto product = [&](const Square<R>& a, const Square<R>& b) {
    return multiply64<R>(tid, R, [&](int r, int k) { return a.v[r][k]; }, [&](int k, int c) { return b.v[k][c]; });
  };
  for (int st = 0; st < steps.n; ++st) {
    const double a = steps.c[st][0], b = steps.c[st][1], c = steps.c[st][2];
    each64<R>(tid, product(A, A), [&](int i, int j, double v) { P.v[i][j] = (i == j ? a : 0.0) + b * A.v[i][j] + c * v; });
    __syncthreads();
    const bool more = st + 1 < steps.n;
    const d4 q = product(P, Q), t = more ? product(P, A) : d4{};
    __syncthreads();
    each64<R>(tid, q, [&](int i, int j, double v) { Q.v[i][j] = v; });
    if (more) {
      each64<R>(tid, t, [&](int i, int j, double v) { T.v[i][j] = v; });
      __syncthreads();
      each64<R>(tid, product(T, P), [&](int i, int j, double v) { A.v[i][j] = v; });
    }
    __syncthreads();
  }
  for (int e = tid; e < R * R; e += kThreads64<R>) Q.v[e / R][e % R] *= inv;
  __syncthreads();
}
// out = Q t for the chunk's columns: a wave per 16 columns at a time
template <int R, class T>
__device__ __forceinline__ void apply64(const Square<R>& Q, const Columns<R>& t, T* dst, int64_t old, int m, int w, int j0,
                                        bool tall, int tid) {
  const int l = tid & 63, wv = tid >> 6, i = l & 15, g = l >> 4;
  for (int c = 16 * wv; c < w; c += kThreads64<R> / 4)
#pragma unroll
    for (int r = 0; r < R; r += 16) {
      if (r >= m) break;
      d4 acc = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
      for (int k = 0; k < R; k += 4)
        acc = __builtin_amdgcn_mfma_f64_16x16x4f64(Q.v[r + i][k + g], (double)t.v[k + g][c + i], acc, 0, 0, 0);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int row = r + g + 4 * q, col = j0 + c + i;
        if (row >= m || c + i >= w) continue;
        const T v = (T)(float)acc[q];
        if (tall) dst[(int64_t)col * old + row] = v;
        else dst[(int64_t)row * old + col] = v;
      }
    }
}

// Matrices of at most kGramChunk columns: all of it in one launch, a block each
template <class T, int R>
__global__ void __launch_bounds__(kThreads64<R>)
ns_small64_kernel(const T* g, int64_t stride, int64_t ld, int m, int n, bool tall, double eps, NsSteps steps, T* out,
                  int64_t ostride, int64_t old) {
  __shared__ Square<R> A, P, Q, S;
  __shared__ Columns<R> t;
  __shared__ double s_inv;
  const int tid = threadIdx.x;
  load_columns<R>(t, g + (int64_t)blockIdx.x * stride, ld, m, n, 0, tall, tid);
  __syncthreads();
  each64<R>(tid, gram64<R>(t, n, tid), [&](int i, int j, double v) { A.v[i][j] = v; });
  __syncthreads();
  iterate64<R>(A, P, Q, S, s_inv, eps, steps, tid);
  apply64<R>(Q, t, out + (int64_t)blockIdx.x * ostride, old, m, n, 0, tall, tid);
}
// Longer ones: partial sums of A per chunk of columns, the iteration, the product per chunk
template <class T, int R>
__global__ void __launch_bounds__(kThreads64<R>) ns_gram64_kernel(const T* __restrict__ g, int64_t stride, int64_t ld, int m, int n,
                                                        bool tall, double* __restrict__ part) {
  __shared__ Columns<R> t;
  const int tid = threadIdx.x, j0 = blockIdx.x * kGramChunk;
  load_columns<R>(t, g + (int64_t)blockIdx.y * stride, ld, m, n, j0, tall, tid);
  __syncthreads();
  double* o = part + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * R * R;
  each64<R>(tid, gram64<R>(t, min(kGramChunk, n - j0), tid), [&](int i, int j, double v) { o[i * R + j] = v; });
}
template <int R>
__global__ void __launch_bounds__(kThreads64<R>)
ns_iterate64_kernel(const double* __restrict__ part, int chunks, double eps, NsSteps steps, double* __restrict__ q) {
  __shared__ Square<R> A, P, Q, S;
  __shared__ double s_inv;
  const int tid = threadIdx.x;
  const double* p = part + (int64_t)blockIdx.x * chunks * R * R;
  for (int e = tid; e < R * R; e += kThreads64<R>) {
    double s = 0.0;
    for (int c = 0; c < chunks; ++c) s += p[(int64_t)c * R * R + e];
    A.v[e / R][e % R] = s;
  }
  __syncthreads();
  iterate64<R>(A, P, Q, S, s_inv, eps, steps, tid);
  for (int e = tid; e < R * R; e += kThreads64<R>) q[(int64_t)blockIdx.x * R * R + e] = Q.v[e / R][e % R];
}
template <class T, int R>
__global__ void __launch_bounds__(kThreads64<R>) ns_apply64_kernel(const T* g, int64_t stride, int64_t ld, int m, int n, bool tall,
                                                         const double* __restrict__ q, T* out, int64_t ostride, int64_t old) {
  __shared__ Square<R> Q;
  __shared__ Columns<R> t;
  const int tid = threadIdx.x, j0 = blockIdx.x * kGramChunk;
  for (int e = tid; e < R * R; e += kThreads64<R>) Q.v[e / R][e % R] = q[(int64_t)blockIdx.y * R * R + e];
  load_columns<R>(t, g + (int64_t)blockIdx.y * stride, ld, m, n, j0, tall, tid);
  __syncthreads();
  apply64<R>(Q, t, out + (int64_t)blockIdx.y * ostride, old, m, min(kGramChunk, n - j0), j0, tall, tid);
}

// ------------------------------------------------------------------ matrices that fit LDS
// Up to 128 x 128: one block per matrix does everything, x and A (then B) staying
// in LDS as pairs, padded to MM x NN. Both products of x read the one layout
// [i][j]: rows by ds_read_b128, columns by ds_read_b64_tr_b16; the 16-byte chunks
// of row i are XORed with its three low bits rotated, which keeps eight rows' chunks
// (b128) and four rows' pairs of chunks (transposed) apart. One launch in place of 17:
// 64 x 64 15 us, 128 x 128 53 us for one matrix or for thirty: LDS is busy for 54 % of
// that (half of it bank conflicts), the matrix pipes for 28 %.
template <int LD>
__device__ __forceinline__ int fit_chunk(int i, int j) {
  return i * LD + (((j >> 3) ^ (((i & 3) << 1) | ((i >> 2) & 1))) << 3);
}
// (a fragment's chunk is (k / 8 + lane / 16) ^ swizzle with k a multiple of 32: one
// XOR of k onto the lane's place at k = 0)
template <int LD>
__device__ __forceinline__ us8 fit_rows(const unsigned short* t, int row0, int k0, int lane) {
  return *reinterpret_cast<const us8*>(t + (fit_chunk<LD>(row0 + (lane & 15), 8 * (lane >> 4)) ^ k0));
}
template <int LD>
__device__ __forceinline__ us8 fit_cols(const unsigned short* t, int col0, int k0, int lane) {
  typedef __attribute__((address_space(3))) s4 lds_s4;
  typedef short s8_ __attribute__((ext_vector_type(8)));
  const int i = lane & 15, k = 8 * (lane >> 4) + (i >> 2), c = col0 + 4 * (i & 3);
  const unsigned short* p = t + k0 * LD;   // (k0 does not change the swizzle)
  const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(p + fit_chunk<LD>(k, c) + (c & 7)));
  const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(p + fit_chunk<LD>(k + 4, c) + (c & 7)));
  const s8_ r = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  return __builtin_bit_cast(us8, r);
}

// D (R x C) = P Q over K on a 4 x 4 grid of waves; the lane's results in
// acc[j][i]: row 16 i + l%16 and columns 16 j + 4 (l/16) + 0..3 of its wave's
// part. QC: Q[k][c] is x itself, else Q = src^T and its columns are src's rows. SYM:
// D is symmetric: the ten waves of the lower triangle of parts work, the others'
// parts are mirrored by the caller.
constexpr int kFitThreads = 1024;
template <int R, int C, int K, int LDP, int LDQ, bool QC, bool SYM>
struct FitProduct {
  static constexpr int TI = R / 64, TJ = C / 64;
  f4 acc[TJ][TI];
  int r0, c0;
  bool on;
  __device__ __forceinline__ void place(int tid) {
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    int wr = w >> 2, wc = w & 3;
    on = true;
    if constexpr (SYM) {
      on = w < 10;
      wr = w < 1 ? 0 : (w < 3 ? 1 : (w < 6 ? 2 : 3));
      wc = w - wr * (wr + 1) / 2;
    }
    r0 = wr * (R / 4);
    c0 = wc * (C / 4);
  }
  __device__ __forceinline__ void run(const unsigned short* p, int plane_p, const unsigned short* q, int plane_q, int tid) {
    const int lane = tid & 63;
    if (!on) return;
#pragma unroll
    for (int j = 0; j < TJ; ++j)
#pragma unroll
      for (int i = 0; i < TI; ++i) acc[j][i] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < K; k += 32) {
      us8 b[TI][2];
#pragma unroll
      for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) b[i][h] = fit_rows<LDP>(p + h * plane_p, r0 + 16 * i, k, lane);
#pragma unroll
      for (int j = 0; j < TJ; ++j) {
        us8 a[2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
          a[h] = QC ? fit_cols<LDQ>(q + h * plane_q, c0 + 16 * j, k, lane) : fit_rows<LDQ>(q + h * plane_q, c0 + 16 * j, k, lane);
        products<HalfPair>(a, b, acc[j]);
      }
    }
  }
  // f(row, column, values, number)
  template <class F>
  __device__ __forceinline__ void each(int tid, F f) const {
    const int lane = tid & 63;
    if (!on) return;
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
      for (int j = 0; j < TJ; ++j) f(r0 + 16 * i + (lane & 15), c0 + 16 * j + 4 * (lane >> 4), acc[j][i], j * TI + i);
  }
};

template <int LD>
__device__ __forceinline__ f4 fit_read(const unsigned short* t, int plane, int i, int j) {
  return read_pair(reinterpret_cast<const _Float16*>(t + fit_chunk<LD>(i, j) + (j & 7)), plane);
}
template <int LD>
__device__ __forceinline__ void fit_write(unsigned short* t, int plane, int i, int j, f4 v) {
  h4 hi, lo;
  split_pair(v, hi, lo);
  unsigned short* p = t + fit_chunk<LD>(i, j) + (j & 7);
  *reinterpret_cast<h4*>(p) = hi;
  *reinterpret_cast<h4*>(p + plane) = lo;
}

// the same at (i, j) .. (i, j + 3) and, where mirror, at the transposed places
template <int LD>
__device__ __forceinline__ void fit_write_symmetric(unsigned short* t, int plane, int i, int j, f4 v, bool mirror) {
  fit_write<LD>(t, plane, i, j, v);
  if (!mirror) return;
  h4 hi, lo;
  split_pair(v, hi, lo);
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    unsigned short* p = t + fit_chunk<LD>(j + c, i) + (i & 7);
    p[0] = __builtin_bit_cast(unsigned short, (_Float16)hi[c]);
    p[plane] = __builtin_bit_cast(unsigned short, (_Float16)lo[c]);
  }
}

template <class T, int MM, int NN>
__global__ void __launch_bounds__(kFitThreads)
ns_fit_kernel(const T* g, int64_t stride, int64_t ld, int m, int n, bool tall, double eps, ScaledSteps steps, T* out,
              int64_t ostride, int64_t old) {
  constexpr int PX = MM * NN, PA = MM * MM, QUADS = MM * NN / 4 / kFitThreads;
  extern __shared__ __align__(16) unsigned short fit_lds[];
  unsigned short *x = fit_lds, *A = fit_lds + 2 * PX;
  __shared__ double red[kFitThreads / 64];
  const int tid = threadIdx.x;
  const T* src = g + (int64_t)blockIdx.x * stride;
  T* dst = out + (int64_t)blockIdx.x * ostride;
  // quads of four columns; lanes run along g's contiguous axis
  auto place = [&](int u, int& i, int& j) {
    const int q = tid + kFitThreads * u;
    i = tall ? q % MM : q / (NN / 4);
    j = 4 * (tall ? q / MM : q % (NN / 4));
  };
  f4 v[QUADS];
  double s = 0.0;
#pragma unroll
  for (int u = 0; u < QUADS; ++u) {
    int i, j;
    place(u, i, j);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      v[u][c] = i < m && j + c < n ? element(src, ld, tall, i, j + c) : 0.f;
      s += (double)v[u][c] * v[u][c];
    }
  }
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
  if ((tid & 63) == 0) red[tid >> 6] = s;
  __syncthreads();
  s = 0.0;
  for (int i = 0; i < kFitThreads / 64; ++i) s += red[i];
  const double inv = kScaleX / (sqrt(s) + eps);
#pragma unroll
  for (int u = 0; u < QUADS; ++u) {
    int i, j;
    place(u, i, j);
#pragma unroll
    for (int c = 0; c < 4; ++c) v[u][c] = (float)(v[u][c] * inv);
    fit_write<NN>(x, PX, i, j, v[u]);
  }
  __syncthreads();
  // a wave's parts of x and A stay with it in FP32; LDS holds what the others multiply
  using Gram = FitProduct<MM, MM, NN, NN, NN, false, true>;
  using Square_ = FitProduct<MM, MM, MM, MM, MM, false, true>;
  using Update = FitProduct<MM, NN, MM, MM, NN, true, false>;
  f4 xr[Update::TI * Update::TJ];
  {
    Update p;
    p.place(tid);
    p.each(tid, [&](int i, int j, f4, int e) { xr[e] = fit_read<NN>(x, PX, i, j); });
  }
  for (int st = 0; st < steps.n; ++st) {
    const float ca = steps.a[st], cu = steps.u[st], cb = steps.b[st], cc = steps.c[st];
    f4 ar[Gram::TI * Gram::TJ];
    {
      Gram p;
      p.place(tid);
      p.run(x, PX, x, PX, tid);
      p.each(tid, [&](int i, int j, f4 r, int e) {
        ar[e] = r * (kScaleA / (kScaleX * kScaleX));
        fit_write_symmetric<MM>(A, PA, i, j, ar[e], p.r0 != p.c0);
      });
    }
    __syncthreads();
    {
      Square_ p;
      p.place(tid);
      p.run(A, PA, A, PA, tid);
      __syncthreads();
      p.each(tid, [&](int i, int j, f4 r, int e) {
        fit_write_symmetric<MM>(A, PA, i, j, cc * r + cb * ar[e], p.r0 != p.c0);
      });
    }
    __syncthreads();
    Update p;
    p.place(tid);
    p.run(A, PA, x, PX, tid);
    p.each(tid, [&](int i, int j, f4 r, int e) { xr[e] = cu * r + ca * xr[e]; });
    if (st + 1 < steps.n) {
      __syncthreads();
      p.each(tid, [&](int i, int j, f4, int e) { fit_write<NN>(x, PX, i, j, xr[e]); });
      __syncthreads();
    } else {
      p.each(tid, [&](int i, int j, f4, int e) {
        if (i >= m) return;
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (j + c < n) {
            const T r = (T)(xr[e][c] * (1.f / kScaleX));
            if (tall) dst[(int64_t)(j + c) * old + i] = r;
            else dst[(int64_t)i * old + j + c] = r;
          }
      });
    }
  }
}

// ------------------------------------------------------------------ products

// operand of matrix b from element `at`
__device__ __forceinline__ Operand<HalfPair> operand(const PairMat& m, int b, int64_t at, int rows) {
  return {m.p + b * m.stride + at, m.ld, rows, m.plane};
}

// Tile (tm, tn) of the lower triangle in tiles R times as high as wide: R (tm + 1)
// tiles in row tm of tiles
template <int R>
__device__ __forceinline__ void triangle(int t, int& tm, int& tn) {
  tm = (int)((sqrtf(8.f * (t / R) + 1.f) - 1.f) * 0.5f);
  while (R * (tm + 1) * (tm + 2) / 2 <= t) ++tm;
  while (R * tm * (tm + 1) / 2 > t) --tm;
  tn = t - R * tm * (tm + 1) / 2;
}

// out = A = x x^T (POLY false, src = x), or out = B = b A + c A A (src = A), for the
// lower triangle of tiles; the upper one is its mirror. Two 2048 x 2048: 87 and 90 us,
// 0.6 PFLOP/s of the half that is computed (272 blocks on 256 CUs).
template <class S, bool POLY>
__global__ void __launch_bounds__(S::NT) ns_symmetric_kernel(PairMat src, PairMat out, int m, int K, int tiles,
                                                             float ca, float cp) {
  __shared__ __align__(16) unsigned short lds[tile_lds<HalfPair, S>];
  const int tid = threadIdx.x;
  const int id = xcd_order(blockIdx.x, gridDim.x), b = id / tiles;
  int tm, tn;
  constexpr int R = S::BM / S::BN;
  triangle<R>(id - b * tiles, tm, tn);
  const int r0 = tm * S::BM, c0 = tn * S::BN;
  if (c0 >= m) return;   // (the last row of tiles may be short)
  f4 acc[S::TN][S::TM];
  tile_gemm_direct<HalfPair, S, true, true>(operand(src, b, (int64_t)r0 * src.ld, m - r0),
                                            operand(src, b, (int64_t)c0 * src.ld, m - c0), K, lds, tid, acc);
  _Float16* o = out.p + b * out.stride;
  const _Float16* a = src.p + b * src.stride;
  for_results<S, 8, false>(acc, min(S::BM, m - r0), min(S::BN, m - c0), tid, [&](int i, int j, f8 v, int k) {
    const int64_t at = (int64_t)(r0 + i) * out.ld + c0 + j;
    v *= cp;
    if constexpr (POLY) v += ca * read_pair<8>(a + at, src.plane);   // (A and B have the same pitch)
    h8 hi, lo;
    split_pair(v, hi, lo);
    if (k == 8) {
      *reinterpret_cast<h8*>(o + at) = hi;
      *reinterpret_cast<h8*>(o + at + out.plane) = lo;
    } else {
      for (int q = 0; q < k; ++q) {
        o[at + q] = hi[q];
        o[at + out.plane + q] = lo[q];
      }
    }
    if (tn < R * tm)   // below the diagonal blocks
#pragma unroll
      for (int q = 0; q < 8; ++q)
        if (q < k) {
          const int64_t t = (int64_t)(c0 + j + q) * out.ld + r0 + i;
          o[t] = hi[q];
          o[t + out.plane] = lo[q];
        }
  });
}

// x <- a x + B x, as pairs, or the last step's result in its own type and layout. Two
// 2048 x 2048: 99 us (1.04 PFLOP/s), bound by the products; 515 x 211 and smaller by a
// tile's own chain of loads and products.
template <class S, class O>
__global__ void __launch_bounds__(S::NT)
ns_update_kernel(PairMat B, PairMat x, PairMat xo, int m, int n, float ca, float cp, O* out, int64_t ostride,
                 int64_t old, bool tall) {
  __shared__ __align__(16) unsigned short lds[tile_lds<HalfPair, S>];
  const int tid = threadIdx.x;
  const int tiles_n = (x.ld + S::BN - 1) / S::BN, tiles_m = (m + S::BM - 1) / S::BM;
  int id = xcd_order(blockIdx.x, gridDim.x);
  const int b = id / (tiles_n * tiles_m);
  id -= b * tiles_n * tiles_m;
  const int r0 = id / tiles_n * S::BM, c0 = id % tiles_n * S::BN;
  f4 acc[S::TN][S::TM];
  tile_gemm_direct<HalfPair, S, true, false>(operand(B, b, (int64_t)r0 * B.ld, m - r0), operand(x, b, c0, x.ld - c0), m,
                                             lds, tid, acc);
  const _Float16* xi = x.p + b * x.stride;
  for_results<S, 8, true>(acc, min(S::BM, m - r0), min(S::BN, x.ld - c0), tid, [&](int i, int j, f8 v, int k) {
    const int64_t at = (int64_t)(r0 + i) * x.ld + c0 + j;   // (whole vectors: the pitch is a multiple of 8)
    v = cp * v + ca * read_pair<8>(xi + at, x.plane);
    if (out) {
      v *= 1.f / kScaleX;
      O* o = out + b * ostride;
      if (!tall) {
        store_n(o + (int64_t)(r0 + i) * old + c0 + j, v, min(8, n - c0 - j), false);
      } else {
#pragma unroll
        for (int q = 0; q < 8; ++q)
          if (c0 + j + q < n) o[(int64_t)(c0 + j + q) * old + r0 + i] = (O)v[q];
      }
    } else {
      h8 hi, lo;
      split_pair(v, hi, lo);
      _Float16* o = xo.p + b * xo.stride + at;
      *reinterpret_cast<h8*>(o) = hi;
      *reinterpret_cast<h8*>(o + xo.plane) = lo;
    }
  });
}

// ------------------------------------------------------------------ host
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
mace_status launched() { return hipGetLastError() == hipSuccess ? MACE_OK : MACE_EHIP; }

mace_status check(const mace_orthogonalise_desc* d) {
  if (!d || d->batch < 0 || d->rows < 1 || d->cols < 1 || d->n_steps < 0 || d->n_steps > kMaxSteps || !(d->eps >= 0))
    return MACE_EINVAL;
  if (d->dtype < MACE_TYPE_FP32 || d->dtype > MACE_TYPE_FP16) return MACE_EINVAL;
  if (d->ld_g < d->cols || d->ld_out < d->cols || d->stride_g < 0 || d->stride_out < 0) return MACE_EINVAL;
  if (d->batch > 1 && d->stride_out < (int64_t)(d->rows - 1) * d->ld_out + d->cols) return MACE_EINVAL;
  if (d->rows > (1 << 15) || d->cols > (1 << 15) || d->batch > 65535 ||
      (double)d->batch * d->rows * d->cols > 17179869184.0)
    return MACE_EUNSUPPORTED;
  return MACE_OK;
}

// Over the singular values that can occur, s with l = s^2, for x <- P(l) x per step,
// P = a + b l + c l^2: whether every step keeps its operands in range (mace.h), the steps
// on operands scaled to that range, and how far a rounding error of A, relative to A's
// largest eigenvalue, can grow over the steps.
struct StepRange {
  bool ok;
  double growth;
  ScaledSteps scaled;
};
// the power of two, at most 2^60, that takes a value below 1 to 1/2 .. 1
int raise_of(double v) {
  int e;
  std::frexp(v, &e);
  return std::min(60, std::max(0, -e));
}
StepRange range_of(const double* k, int steps) {
  double r = 1.0;   // largest singular value so far
  int up = 0;       // x is scaled by kScaleX 2^up
  StepRange out{true, 1.0, {}};
  out.scaled.n = steps;   // (steps after one that leaves zeros: zeros)
  for (int s = 0; s < steps; ++s, k += 3) {
    const double a = k[0], b = k[1], c = k[2];
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return {};
    double top = 0.0, next = 0.0, p = 0.0, slope = 0.0;
    auto at = [&](double l) {   // l clamped to the range: a point outside gives its end
      l = std::min(std::max(l, 0.0), r * r);
      const double B = b * l + c * l * l;
      top = std::max(top, std::fabs(B));
      next = std::max(next, std::fabs(a + B) * std::sqrt(l));
      p = std::max(p, std::fabs(a + B));
      slope = std::max(slope, std::fabs(a + 3.0 * b * l + 5.0 * c * l * l));
    };
    // the ends of the range, and where the derivatives vanish
    at(0.0);
    at(r * r);
    if (c != 0.0) {
      at(-b / (2.0 * c));
      at(-3.0 * b / (10.0 * c));
      const double d = 9.0 * b * b - 20.0 * a * c;   // a + 3 b l + 5 c l^2 = 0
      if (d >= 0.0) {
        at((-3.0 * b + std::sqrt(d)) / (10.0 * c));
        at((-3.0 * b - std::sqrt(d)) / (10.0 * c));
      }
    } else if (b != 0.0) {
      at(-a / (3.0 * b));
    }
    const double before = r;
    r = next * 1.001;   // (rounding)
    if (!(top <= kMaxB) || !(r <= kMaxSigma)) return {};
    if (r == 0.0) break;   // zeros from here on
    // d(l P^2) / dl = P (P + 2 l P'); each step adds a rounding of its own
    out.growth = out.growth * p * slope * (before / r) * (before / r) + 1.0;
    // (the last step's result leaves at kScaleX, in FP32)
    const int up_next = s + 1 < steps ? raise_of(r) : 0, up_b = top > 0.0 ? raise_of(top) : 0;
    const double sa = std::ldexp(kScaleA, 2 * up), sb = std::ldexp(kScaleB, up_b);
    out.scaled.a[s] = (float)std::ldexp(a, up_next - up);
    out.scaled.u[s] = (float)std::ldexp(1.0 / sb, up_next - up);
    out.scaled.b[s] = (float)(b * (sb / sa));
    out.scaled.c[s] = (float)(c * (sb / sa) / sa);
    up = up_next;
  }
  return out;
}

struct NsPlan {
  int m, n, mp, np, parts;   // parts: partial sums of the norm, or chunks of the FP64 products
  bool tall, gram, fit;   // which of the kernels above; neither: products by launches of tiles
  size_t part, q, x0, x1, A, B, total;
};
NsPlan plan(const mace_orthogonalise_desc& d, double growth) {
  NsPlan p{};
  p.tall = d.rows > d.cols;
  p.m = std::min(d.rows, d.cols);
  p.n = std::max(d.rows, d.cols);
  p.mp = (p.m + 7) / 8 * 8;
  p.np = (p.n + 7) / 8 * 8;
  p.gram = (p.m <= kGramMax || (p.m <= kGramMaxLong && p.n > kFitMax)) && growth <= kGramGrowth;
  p.parts = p.gram ? (int)ceil_div(p.n, kGramChunk) : (int)std::min<int64_t>(kNormBlocks, ceil_div(d.rows, 4));
  p.fit = !p.gram && p.n <= kFitMax;
  size_t o = 0;
  auto take = [&](size_t bytes) {
    const size_t at = o;
    o += (bytes + 255) & ~size_t(255);
    return at;
  };
  if (p.gram) {
    const int r = p.m <= 16 ? 16 : (p.m <= 32 ? 32 : 64);
    if (p.parts > 1 || r == 64) {
      p.part = take(sizeof(double) * d.batch * p.parts * r * r);
      p.q = take(sizeof(double) * d.batch * r * r);
    }
    p.total = o;
    return p;
  }
  if (p.fit && d.n_steps > 0) return p;
  p.part = take(sizeof(double) * d.batch * p.parts);
  p.x0 = take(size_t(4) * d.batch * p.m * p.np);
  p.x1 = take(size_t(4) * d.batch * p.m * p.np);
  p.A = take(size_t(4) * d.batch * p.m * p.mp);
  p.B = take(size_t(4) * d.batch * p.m * p.mp);
  p.total = o;
  return p;
}

constexpr int64_t kFillBlocks = 256;   // (one per CU)

// Mid: 128 x 128, from one block per CU on. Half: the symmetric products' blocks, half
// as wide, where Mid gives less than one per CU and Half that many: there are few of them,
// one triangle's (two 1500 x 1500 752 us, with Small 820; four 1000 x 2000 750 against 817;
// but thirty 300 x 515, whose last tiles are mostly empty, 305 against 278). With a Mid
// block per CU Half takes 9 to 13 % more, as it reads more LDS per product (two 2048 x 2048
// 1440 us against 1315, one 2900 x 2905 2700 against 2400).
using Mid = TileShape<128, 128, 2, 2, 32, 2, true>;
using Half = TileShape<128, 64, 2, 2, 32, 2, true>;
using Small = TileShape<64, 64, 2, 2, 32, 4, true>;

template <bool POLY>
mace_status symmetric(const PairMat& src, const PairMat& out, int64_t batch, int m, int K, float ca, float cp,
                      hipStream_t s) {
  auto go = [&](auto shape) {
    using S = decltype(shape);
    const int64_t t = ceil_div(m, S::BM), tiles = S::BM / S::BN * t * (t + 1) / 2;
    ns_symmetric_kernel<S, POLY><<<(unsigned)(tiles * batch), S::NT, 0, s>>>(src, out, m, K, (int)tiles, ca, cp);
    return launched();
  };
  const int64_t t = ceil_div(m, 128);
  if (t * (t + 1) / 2 * batch >= kFillBlocks) return go(Mid{});
  return t * (t + 1) * batch >= kFillBlocks ? go(Half{}) : go(Small{});
}
template <class O>
mace_status update(const PairMat& B, const PairMat& x, const PairMat& xo, int64_t batch, int m, int n, float ca, float cp,
                   O* out, int64_t ostride, int64_t old, bool tall, hipStream_t s) {
  auto go = [&](auto shape) {
    using S = decltype(shape);
    const int64_t blocks = ceil_div(m, S::BM) * ceil_div(x.ld, S::BN) * batch;
    ns_update_kernel<S, O><<<(unsigned)blocks, S::NT, 0, s>>>(B, x, xo, m, n, ca, cp, out, ostride, old, tall);
    return launched();
  };
  return ceil_div(m, 128) * ceil_div(x.ld, 128) * batch >= kFillBlocks ? go(Mid{}) : go(Small{});
}

template <class O, int MM, int NN>
mace_status run_fit(const mace_orthogonalise_desc& d, const NsPlan& p, const ScaledSteps& steps, const O* g, O* out,
                    hipStream_t s) {
  constexpr int bytes = 2 * 2 * (MM * NN + MM * MM);
  auto f = ns_fit_kernel<O, MM, NN>;
  if (bytes > 65536 && hipFuncSetAttribute(reinterpret_cast<const void*>(f), hipFuncAttributeMaxDynamicSharedMemorySize,
                                           bytes) != hipSuccess)
    return MACE_EHIP;
  f<<<(unsigned)d.batch, kFitThreads, bytes, s>>>(g, d.stride_g, d.ld_g, p.m, p.n, p.tall, d.eps, steps, out, d.stride_out,
                                          d.ld_out);
  return launched();
}

template <class O>
mace_status run(const mace_orthogonalise_desc& d, const NsPlan& p, const ScaledSteps& scaled, const O* g,
                const double* coef, O* out, char* ws, hipStream_t s) {
  double* part = reinterpret_cast<double*>(ws + p.part);
  mace_status st;
  if (p.fit && d.n_steps > 0) {
    if (p.n <= 64) return run_fit<O, 64, 64>(d, p, scaled, g, out, s);
    if (p.m <= 64) return run_fit<O, 64, 128>(d, p, scaled, g, out, s);
    return run_fit<O, 128, 128>(d, p, scaled, g, out, s);
  }
  if (p.gram) {
    NsSteps steps{};
    steps.n = d.n_steps;
    for (int i = 0; i < 3 * d.n_steps; ++i) steps.c[i / 3][i % 3] = coef[i];
    auto go = [&](auto r_) -> mace_status {
      constexpr int R = decltype(r_)::value;
      if constexpr (R <= 32) if (p.parts == 1) {
        ns_small64_kernel<O, R><<<(unsigned)d.batch, 256, 0, s>>>(g, d.stride_g, d.ld_g, p.m, p.n, p.tall, d.eps, steps,
                                                                  out, d.stride_out, d.ld_out);
        return launched();
      }
      double* q = reinterpret_cast<double*>(ws + p.q);
      const dim3 grid(p.parts, (unsigned)d.batch);
      constexpr int NT = kThreads64<R>;
      ns_gram64_kernel<O, R><<<grid, NT, 0, s>>>(g, d.stride_g, d.ld_g, p.m, p.n, p.tall, part);
      if ((st = launched()) != MACE_OK) return st;
      ns_iterate64_kernel<R><<<(unsigned)d.batch, NT, 0, s>>>(part, p.parts, d.eps, steps, q);
      if ((st = launched()) != MACE_OK) return st;
      ns_apply64_kernel<O, R><<<grid, NT, 0, s>>>(g, d.stride_g, d.ld_g, p.m, p.n, p.tall, q, out, d.stride_out, d.ld_out);
      return launched();
    };
    return p.m <= 16 ? go(Int<16>{}) : (p.m <= 32 ? go(Int<32>{}) : go(Int<64>{}));
  }
  ns_norm_kernel<O><<<dim3(p.parts, (unsigned)d.batch), 256, 0, s>>>(g, d.stride_g, d.ld_g, d.rows, d.cols, part);
  if ((st = launched()) != MACE_OK) return st;
  if (d.n_steps == 0) {
    ns_scale_kernel<O><<<dim3((unsigned)ceil_div((int64_t)d.rows * d.cols, 256), (unsigned)d.batch), 256, 0, s>>>(
        g, d.stride_g, d.ld_g, d.rows, d.cols, part, p.parts, d.eps, out, d.stride_out, d.ld_out);
    return launched();
  }
  auto mat = [&](size_t at, int ld) {
    const int64_t plane = (int64_t)p.m * ld;
    return PairMat{reinterpret_cast<_Float16*>(ws + at), 2 * plane, plane, ld};
  };
  PairMat x = mat(p.x0, p.np), xo = mat(p.x1, p.np);
  const PairMat A = mat(p.A, p.mp), B = mat(p.B, p.mp);
  ns_pack_kernel<O><<<dim3((unsigned)ceil_div(p.np, 64), (unsigned)ceil_div(p.m, 64), (unsigned)d.batch), 256, 0, s>>>(
      g, d.stride_g, d.ld_g, p.m, p.n, p.tall, part, p.parts, d.eps, x, A, B);
  if ((st = launched()) != MACE_OK) return st;
  for (int i = 0; i < d.n_steps; ++i) {
    constexpr float g = kScaleA / (kScaleX * kScaleX);
    O* o = i == d.n_steps - 1 ? out : nullptr;
    if ((st = symmetric<false>(x, A, d.batch, p.m, p.np, 0.f, g, s)) != MACE_OK) return st;
    if ((st = symmetric<true>(A, B, d.batch, p.m, p.m, scaled.b[i], scaled.c[i], s)) != MACE_OK) return st;
    if ((st = update<O>(B, x, xo, d.batch, p.m, p.n, scaled.a[i], scaled.u[i], o, d.stride_out, d.ld_out, p.tall, s)) !=
        MACE_OK)
      return st;
    std::swap(x, xo);
  }
  return MACE_OK;
}

}  // namespace
}  // namespace mace

using namespace mace;

extern "C" size_t mace_orthogonalise_workspace_bytes(const mace_orthogonalise_desc* desc) {
  if (check(desc) != MACE_OK) return 0;
  return std::max(plan(*desc, 1.0).total, plan(*desc, INFINITY).total) + 256;   // (whatever the coefficients)
}

extern "C" mace_status mace_orthogonalise(const mace_orthogonalise_desc* desc, const void* g, const double* coefficients,
                                          void* out, void* workspace, size_t workspace_bytes, void* stream) {
  const mace_status st = check(desc);
  if (st != MACE_OK) return st;
  if (desc->n_steps > 0 && !coefficients) return MACE_EINVAL;
  if (desc->batch == 0) return MACE_OK;
  if (!g || !out || !workspace) return MACE_EINVAL;
  const StepRange range = range_of(coefficients, desc->n_steps);
  if (!range.ok) return MACE_ERANGE;
  if (workspace_bytes < mace_orthogonalise_workspace_bytes(desc)) return MACE_ENOSPACE;
  char* ws = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(workspace) + 255) & ~uintptr_t(255));
  const NsPlan p = plan(*desc, range.growth);
  hipStream_t s = (hipStream_t)stream;
  if (desc->dtype == MACE_TYPE_FP32) return run<float>(*desc, p, range.scaled, (const float*)g, coefficients, (float*)out, ws, s);
  if (desc->dtype == MACE_TYPE_BF16)
    return run<__bf16>(*desc, p, range.scaled, (const __bf16*)g, coefficients, (__bf16*)out, ws, s);
  return run<_Float16>(*desc, p, range.scaled, (const _Float16*)g, coefficients, (_Float16*)out, ws, s);
}
