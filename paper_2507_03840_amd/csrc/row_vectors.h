// Rows read and written in vectors of 16 bytes (or 8), whatever their length and alignment, by lanes that keep a vector as it lies in memory.
#pragma once
#include "row_types.h"

template <class T> struct RvWidth { static constexpr int V = 16 / sizeof(T); };

// v moved down by `by` words, zeros behind (any by >= 0; words moved by 1, 2 and 4 of them, each where its bit is set)
template <int W>
__device__ __forceinline__ void rv_move_words(unsigned (&v)[W], int by) {
#pragma unroll
  for (int step = 1; step < W; step *= 2)
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = by & step ? (i + step < W ? v[i + step] : 0u) : v[i];
#pragma unroll
  for (int i = 0; i < W; ++i) v[i] = by >= W ? 0u : v[i];
}

// EVEN: every row begins at a multiple of 16 bytes and is a multiple of 16 bytes long.  Otherwise vectors are aligned to a value only, and
// the last one of a row may be a part: the row's last V values are read in its place and moved down by the values too many (loads are never under a
// condition, as they would be waited for one by one); what is written of it goes value by value.  Rows of V values at least, but for load_any.
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
      constexpr int W = V * (int)sizeof(T) / 4;
      const int at = min(j * V, n - V), over = j * V - at;
      const loose u = *(const loose*)(row + at);
      unsigned w[W];
      __builtin_memcpy(w, &u, sizeof(w));
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = over & 1 ? __builtin_amdgcn_alignbit(i + 1 < W ? w[i + 1] : 0u, w[i], 16) : w[i];
        rv_move_words(w, over >> 1);
      } else {
        rv_move_words(w, over);
      }
      vec v;
      __builtin_memcpy(&v, w, sizeof(w));
      return v;
    }
  }
  static __device__ __forceinline__ vec load_any(const T* row, int j, int n) {
    if (EVEN || n >= V) return load(row, j, n);
    vec v = {};
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (j * V + i < n) v[i] = row[j * V + i];
    return v;
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
      typedef float floats __attribute__((ext_vector_type(V)));
      typedef floats loose_floats __attribute__((aligned(4)));
      const int at = min(j * V, n - V);
      const loose_floats u = *(const loose_floats*)(row + at);
      unsigned w[V];
      __builtin_memcpy(w, &u, sizeof(w));
      rv_move_words(w, j * V - at);
      __builtin_memcpy(v, w, sizeof(w));
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
