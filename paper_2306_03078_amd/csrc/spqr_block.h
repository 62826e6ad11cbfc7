// Shared by spqr_norm.hip, spqr_adapter.hip and spqr_score.hip: runs of elements at any address, sums over a workgroup, checks.
#ifndef SPQR_BLOCK_INTERNAL_H_
#define SPQR_BLOCK_INTERNAL_H_
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/spqr_block.h"
#include "spqr_device.h"

namespace spqr_blk {

using spqr::u32x4;

inline bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
inline bool known(int dtype) { return dtype == SPQR_F32 || dtype == SPQR_F16 || dtype == SPQR_BF16; }
inline size_t size_of(int dtype) { return dtype == SPQR_F32 ? 4 : 2; }
inline int launched() { return hipGetLastError() == hipSuccess ? SPQR_OK : SPQR_ERR_HIP; }

// Eight neighbouring elements, at any address that one of them may have: the card's wide loads and stores take these (rows of odd
// width begin anywhere).
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Run8 { T e[8]; };

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
  const Run8<T> r = *reinterpret_cast<const Run8<T>*>(p);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (float)r.e[e];
}

// Elements at .. at + 7 of a row of n; zeros behind its end.
template <typename T>
__device__ __forceinline__ void load_row8(const T* row, int at, int n, float (&v)[8]) {
  if (at + 8 <= n) {
    load8(row + at, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = at + e < n ? (float)row[at + e] : 0.f;
  }
}

__device__ __forceinline__ void load_row8_as(int dtype, const void* row, int64_t from, int at, int n, float (&v)[8]) {
  if (dtype == SPQR_F32) load_row8(static_cast<const float*>(row) + from, at, n, v);
  else if (dtype == SPQR_F16) load_row8(static_cast<const _Float16*>(row) + from, at, n, v);
  else load_row8(static_cast<const __bf16*>(row) + from, at, n, v);
}

template <typename T>
__device__ __forceinline__ void store_row8(T* row, int at, int n, const float (&v)[8]) {
  if (at + 8 <= n) {
    Run8<T> r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r.e[e] = (T)v[e];
    *reinterpret_cast<Run8<T>*>(row + at) = r;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (at + e < n) row[at + e] = (T)v[e];
  }
}

__device__ __forceinline__ void store_row8_as(int dtype, void* row, int64_t from, int at, int n, const float (&v)[8]) {
  if (dtype == SPQR_F32) store_row8(static_cast<float*>(row) + from, at, n, v);
  else if (dtype == SPQR_F16) store_row8(static_cast<_Float16*>(row) + from, at, n, v);
  else store_row8(static_cast<__bf16*>(row) + from, at, n, v);
}

}  // namespace spqr_blk
#endif
