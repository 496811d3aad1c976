// Runs of N elements as one load (of 4, 8 or 16 bytes) or store (of 8 or 16) where they fill it, element by element otherwise.
#pragma once
#include "common.h"

namespace cd {

template <typename T, int N> __device__ static inline void load_run(const T* p, T (&out)[N]) {
  if constexpr (N * sizeof(T) == 16) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    __builtin_memcpy(out, &u, 16);
  } else if constexpr (N * sizeof(T) == 8) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    __builtin_memcpy(out, &u, 8);
  } else if constexpr (N * sizeof(T) == 4) {
    const uint32_t u = *reinterpret_cast<const uint32_t*>(p);
    __builtin_memcpy(out, &u, 4);
  } else {
#pragma unroll
    for (int i = 0; i < N; i++) out[i] = p[i];
  }
}
// the same from an address that is whole in its elements only: the same instructions, which global memory takes at any address
typedef uint32_t run4_t __attribute__((ext_vector_type(4)));
typedef uint32_t run4_anywhere_t __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t run2_anywhere_t __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t run1_anywhere_t __attribute__((aligned(2)));
template <typename T, int N> __device__ static inline void load_run_anywhere(const T* p, T (&out)[N]) {
  if constexpr (N * sizeof(T) == 16) {
    const run4_t u = *reinterpret_cast<const run4_anywhere_t*>(p);
    __builtin_memcpy(out, &u, 16);
  } else if constexpr (N * sizeof(T) == 8) {
    const run2_anywhere_t u = *reinterpret_cast<const run2_anywhere_t*>(p);
    __builtin_memcpy(out, &u, 8);
  } else if constexpr (N * sizeof(T) == 4) {
    const uint32_t u = *reinterpret_cast<const run1_anywhere_t*>(p);
    __builtin_memcpy(out, &u, 4);
  } else {
#pragma unroll
    for (int i = 0; i < N; i++) out[i] = p[i];
  }
}
// the same past the caches, where 16 bytes are read once (at any address, too)
template <typename T, int N> __device__ static inline void load_run_stream(const T* p, T (&out)[N]) {
  if constexpr (N * sizeof(T) == 16) {
    const run4_t u = __builtin_nontemporal_load(reinterpret_cast<const run4_anywhere_t*>(p));
    __builtin_memcpy(out, &u, 16);
  } else {
    load_run_anywhere<T, N>(p, out);
  }
}
template <typename T, int N> __device__ static inline void store_run_stream(T* p, const float (&in)[N]) {
  if constexpr (N * sizeof(T) == 16) {
    T t[N];
#pragma unroll
    for (int i = 0; i < N; i++) t[i] = Cvt<T>::st(in[i]);
    run4_t u;
    __builtin_memcpy(&u, t, 16);
    __builtin_nontemporal_store(u, reinterpret_cast<run4_t*>(p));
  } else {
#pragma unroll
    for (int i = 0; i < N; i++) p[i] = Cvt<T>::st(in[i]);
  }
}
template <typename T, int N> __device__ static inline void store_run(T* p, const float (&in)[N]) {
  T t[N];
#pragma unroll
  for (int i = 0; i < N; i++) t[i] = Cvt<T>::st(in[i]);
  if constexpr (N * sizeof(T) == 16) {
    uint4 u;
    __builtin_memcpy(&u, t, 16);
    *reinterpret_cast<uint4*>(p) = u;
  } else if constexpr (N * sizeof(T) == 8) {
    uint2 u;
    __builtin_memcpy(&u, t, 8);
    *reinterpret_cast<uint2*>(p) = u;
  } else {
#pragma unroll
    for (int i = 0; i < N; i++) p[i] = t[i];
  }
}

}  // namespace cd
