// Vectors of stored elements (gist_store) as floats: loads that widen, stores
// that round once to nearest even.
#pragma once

#include "common.cuh"
#include "gist_internal.h"

namespace gist {

// Aligned as their elements are: rows of any width and leading dimension are
// moved 16 bytes at a time (the hardware takes any address for global accesses;
// only a lane whose bytes cross a line costs more).
typedef float fx4 __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned short us8 __attribute__((ext_vector_type(8), aligned(2)));

// ---- stored elements as floats ------------------------------------------------

template <int STORE>
__device__ __forceinline__ float widen(unsigned short u) {
  if constexpr (STORE == GIST_STORE_BF16) return __uint_as_float(static_cast<unsigned>(u) << 16);
  return static_cast<float>(__builtin_bit_cast(_Float16, u));
}

template <int STORE, int V>
__device__ __forceinline__ void load_vec(const void* base, int64_t e, float (&x)[V]) {
  if constexpr (STORE == GIST_STORE_F32) {
    const float* p = static_cast<const float*>(base) + e;
    if constexpr (V == 4) {
      const fx4 t = *reinterpret_cast<const fx4*>(p);
#pragma unroll
      for (int q = 0; q < 4; ++q) x[q] = t[q];
    } else {
      static_assert(V == 1, "one float or four");
      x[0] = *p;
    }
  } else {
    const unsigned short* p = static_cast<const unsigned short*>(base) + e;
    if constexpr (V == 8) {
      const us8 t = *reinterpret_cast<const us8*>(p);
#pragma unroll
      for (int q = 0; q < 8; ++q) x[q] = widen<STORE>(t[q]);
    } else {
      static_assert(V == 1, "one 16-bit element or eight");
      x[0] = widen<STORE>(*p);
    }
  }
}

template <int V>
__device__ __forceinline__ void store_vec(float* p, const float (&x)[V]) {
  if constexpr (V == 4 || V == 8) {
#pragma unroll
    for (int h = 0; h < V; h += 4) {
      fx4 t;
#pragma unroll
      for (int q = 0; q < 4; ++q) t[q] = x[h + q];
      *reinterpret_cast<fx4*>(p + h) = t;
    }
  } else {
    static_assert(V == 1, "one float, four or eight");
    *p = x[0];
  }
}

template <int STORE>
__device__ __forceinline__ unsigned short narrow(float x) {
  if constexpr (STORE == GIST_STORE_BF16) return __builtin_bit_cast(unsigned short, static_cast<__bf16>(x));
  return __builtin_bit_cast(unsigned short, static_cast<_Float16>(x));
}

template <int STORE, int V>
__device__ __forceinline__ void store_as(void* base, int64_t e, const float (&x)[V]) {
  if constexpr (STORE == GIST_STORE_F32) {
    store_vec<V>(static_cast<float*>(base) + e, x);
  } else {
    unsigned short* p = static_cast<unsigned short*>(base) + e;
    if constexpr (V == 8) {
      us8 t;
#pragma unroll
      for (int q = 0; q < 8; ++q) t[q] = narrow<STORE>(x[q]);
      *reinterpret_cast<us8*>(p) = t;
    } else {
      static_assert(V == 1, "one 16-bit element or eight");
      *p = narrow<STORE>(x[0]);
    }
  }
}

// Elements e .. e + V - 1, of which the first `left` are there; the others are `fill`.
template <int STORE, int V>
__device__ __forceinline__ void load_some(const void* base, int64_t e, int64_t left, float fill, float (&x)[V]) {
  if (left >= V) {
    load_vec<STORE, V>(base, e, x);
  } else {
#pragma unroll
    for (int q = 0; q < V; ++q) {
      float y[1] = {fill};
      if (q < left) load_vec<STORE, 1>(base, e + q, y);
      x[q] = y[0];
    }
  }
}

template <int STORE, int V>
__device__ __forceinline__ void store_some(void* base, int64_t e, int64_t left, const float (&x)[V]) {
  if (left >= V) {
    store_as<STORE, V>(base, e, x);
  } else {
#pragma unroll
    for (int q = 0; q < V; ++q) {
      const float y[1] = {x[q]};
      if (q < left) store_as<STORE, 1>(base, e + q, y);
    }
  }
}

// Orders a wave's LDS reads and writes before it and after it, whichever lanes make them.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

inline int ceil_log2(int64_t x) {
  int l = 0;
  while ((int64_t{1} << l) < x) ++l;
  return l;
}

}  // namespace gist
