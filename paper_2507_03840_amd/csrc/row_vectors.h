// Rows read and written in vectors of 16 bytes (or 8), whatever their length and alignment, by lanes that keep a vector as it lies in memory.
#pragma once
#include "row_types.h"

template <class T> struct RvWidth { static constexpr int V = 16 / sizeof(T); };

// EVEN: every row begins at a multiple of 16 bytes and is a multiple of 16 bytes long.  Otherwise vectors are aligned to a value only, and
// the last one of a row may be a part, whose values go one by one.
template <class T, bool EVEN, int WIDTH = RvWidth<T>::V>
struct Rv {
  static constexpr int V = WIDTH;
  typedef T vec __attribute__((ext_vector_type(V)));
  typedef vec loose __attribute__((aligned(sizeof(T))));

  // vector j of a row of n values; zeros behind its end.  EVEN: behind the end the last vector (loads are never under a condition)
  static __device__ __forceinline__ vec load(const T* row, int j, int n) {
    if constexpr (EVEN) {
      return *(const vec*)(row + min(j, n / V - 1) * V);
    } else {
      vec v = {};
      if ((j + 1) * V <= n) {
        v = *(const loose*)(row + j * V);
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (j * V + i < n) v[i] = row[j * V + i];
      }
      return v;
    }
  }
  static __device__ __forceinline__ void store(T* row, int j, int n, const vec& v) {
    if constexpr (EVEN) {
      if (j * V < n) *(vec*)(row + j * V) = v;
    } else if ((j + 1) * V <= n) {
      *(loose*)(row + j * V) = v;
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (j * V + i < n) row[j * V + i] = v[i];
    }
  }
  // the same for V floats beside the row
  static __device__ __forceinline__ void load_floats(const float* row, int j, int n, float (&v)[V]) {
    if constexpr (EVEN) {
      typedef float floats __attribute__((ext_vector_type(V)));
      const floats u = *(const floats*)(row + min(j, n / V - 1) * V);
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = u[i];
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = row[min(j * V + i, n - 1)];
    }
  }
};

inline bool rv_aligned(std::initializer_list<const void*> at, std::initializer_list<int64_t> bytes) {
  for (const void* a : at)
    if ((uintptr_t)a % 16) return false;
  for (int64_t b : bytes)
    if (b % 16) return false;
  return true;
}
