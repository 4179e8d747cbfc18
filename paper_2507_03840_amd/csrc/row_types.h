// Rows of fp32, IEEE half precision or bfloat16 (EGNN_F32, EGNN_F16, EGNN_BF16): vectors of V values in and out as fp32.
#pragma once
#include <initializer_list>
#include "egnn_internal.h"

inline int rt_size(int32_t dtype) { return dtype == EGNN_F32 ? 4 : dtype == EGNN_F16 || dtype == EGNN_BF16 ? 2 : 0; }

// Lets a kernel have more than 64 KB of dynamic LDS, once per kernel and GPU (`ready`: a static of the caller; set twice to the same by two threads).
inline int rt_allow_lds(egnn_ctx* ctx, const void* kernel, size_t bytes, bool (&ready)[64]) {
  int device = 0;
  if (bytes <= 65536) return EGNN_OK;
  EGNN_HIP(ctx, hipGetDevice(&device));
  if (device >= 0 && device < 64 && ready[device]) return EGNN_OK;
  EGNN_HIP(ctx, hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
  if (device >= 0 && device < 64) ready[device] = true;
  return EGNN_OK;
}

// V values at p, which is aligned to all of them
template <class T, int V>
__device__ __forceinline__ void rt_load(const T* p, float (&v)[V]) {
  typedef T vec __attribute__((ext_vector_type(V)));
  const vec u = *reinterpret_cast<const vec*>(p);
#pragma unroll
  for (int q = 0; q < V; ++q) v[q] = (float)u[q];
}
template <class T, int V>
__device__ __forceinline__ void rt_store(T* p, const float (&v)[V]) {
  typedef T vec __attribute__((ext_vector_type(V)));
  vec u;
#pragma unroll
  for (int q = 0; q < V; ++q) u[q] = (T)v[q];   // one rounding to nearest even
  *reinterpret_cast<vec*>(p) = u;
}
