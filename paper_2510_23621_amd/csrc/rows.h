// Rows read and written 16 bytes a lane, and the host side that operators on them share.
#pragma once

#include "../../include/mace.h"
#include "dense.h"

namespace mace {

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

// Item block * 256 + threadIdx.x as (row, vector) of rows of nv vectors, with
// one division of 64 bits per block.
__device__ __forceinline__ int64_t item_row(int nv, int& vec, int block) {
  const uint64_t i0 = (uint64_t)block * 256;
  const uint64_t q0 = i0 >> 32 ? i0 / (unsigned)nv : (unsigned)i0 / (unsigned)nv;
  const unsigned j = (unsigned)(i0 - q0 * (unsigned)nv) + threadIdx.x, q = j / (unsigned)nv;
  vec = (int)(j - q * (unsigned)nv);
  return (int64_t)(q0 + q);
}
__device__ __forceinline__ int64_t item_row(int nv, int& vec) { return item_row(nv, vec, block_id()); }

inline mace_status launched() { return hipGetLastError() == hipSuccess ? MACE_OK : MACE_EHIP; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
template <class F>
mace_status by_type(int dtype, F f) {
  if (dtype == MACE_TYPE_FP32) return f(0.f);
  if (dtype == MACE_TYPE_BF16) return f((__bf16)0.f);
  return f((_Float16)0.f);
}

}  // namespace mace
