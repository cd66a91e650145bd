// Rows of fp32, fp16 or bf16 elements: a thread's V consecutive elements as
// fp32 values, read and written in one access where the row allows it.
// Conversions to 16 bits round to nearest even, once, at the store.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dpi.h"

namespace dpi {
namespace {

typedef _Float16 f16_t;
typedef __bf16 bf16_t;

template <typename T, int V>
struct Raw {
  typedef T plain __attribute__((ext_vector_type(V)));
  typedef plain type __attribute__((aligned(sizeof(T) * V < 16 ? sizeof(T) * V : 16)));
};

// The elements as they lie in memory, converted when they are used: a tile of
// raw 16-bit elements takes half the registers of their fp32 values.
template <typename T, int V>
struct Elems {
  typename Raw<T, V>::type raw;
  __device__ __forceinline__ float operator[](int i) const { return (float)raw[i]; }
};

// WIDE: p is aligned to the whole access and all V elements exist.  Otherwise
// element by element, an element past the row's end (i >= have) being read from
// the row's last one: no access leaves the row.
template <bool WIDE, typename T, int V>
__device__ __forceinline__ Elems<T, V> load_elems(const T* p, int have) {
  Elems<T, V> e;
  if constexpr (WIDE) {
    e.raw = *reinterpret_cast<const typename Raw<T, V>::type*>(p);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) e.raw[i] = p[min(i, have - 1)];
  }
  return e;
}

template <bool WIDE, typename T, int V>
__device__ __forceinline__ void store_elems(T* p, const float* v, int have) {
  if constexpr (WIDE) {
    typename Raw<T, V>::type r;
#pragma unroll
    for (int i = 0; i < V; ++i) r[i] = (T)v[i];
    *reinterpret_cast<typename Raw<T, V>::type*>(p) = r;
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < have) p[i] = (T)v[i];
  }
}

// The same, all V there and aligned, past the caches' order of use: rows that nothing reads again soon.
template <typename T, int V>
__device__ __forceinline__ Elems<T, V> load_once(const T* p) {
  Elems<T, V> e;
  e.raw = __builtin_nontemporal_load(reinterpret_cast<const typename Raw<T, V>::type*>(p));
  return e;
}

template <typename T, int V>
__device__ __forceinline__ void store_once(T* p, const float* v) {
  typename Raw<T, V>::plain r;
#pragma unroll
  for (int i = 0; i < V; ++i) r[i] = (T)v[i];
  __builtin_nontemporal_store(r, reinterpret_cast<typename Raw<T, V>::type*>(p));
}

}  // namespace

inline int elem_size(int32_t dtype) { return dtype == DPI_F32 ? 4 : 2; }
inline bool known_dtype(int32_t dtype) { return dtype == DPI_F32 || dtype == DPI_F16 || dtype == DPI_BF16; }

}  // namespace dpi
