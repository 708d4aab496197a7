// Entries in 32 or 16 bits, read as fp32 and rounded once (to nearest even) where they are written.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace choco {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// V entries that one load or store moves.
template <class T, int V>
struct alignas(V * sizeof(T)) Pack {
  T e[V];
};

template <class T>
__device__ __forceinline__ float to_float(T x) { return (float)x; }
template <class T>
__device__ __forceinline__ T from_float(float x) { return (T)x; }

template <class T, int V>
__device__ __forceinline__ void load_floats(const T* p, float (&x)[V]) {
  const Pack<T, V> v = *reinterpret_cast<const Pack<T, V>*>(p);
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = to_float(v.e[i]);
}
template <class T, int V>
__device__ __forceinline__ void store_floats(T* p, const float (&x)[V]) {
  Pack<T, V> v;
#pragma unroll
  for (int i = 0; i < V; ++i) v.e[i] = from_float<T>(x[i]);
  *reinterpret_cast<Pack<T, V>*>(p) = v;
}

// ... past the caches.
template <class T, int V>
__device__ __forceinline__ void store_floats_past(T* p, const float (&x)[V]) {
  typedef T Entries __attribute__((ext_vector_type(V)));
  Entries v;
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = from_float<T>(x[i]);
  __builtin_nontemporal_store(v, reinterpret_cast<Entries*>(p));
}

// Entry i of a register's worth of them.
template <class T>
__device__ __forceinline__ float entry(uint32_t word, int i) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(word);
  else if constexpr (std::is_same_v<T, bf16_t>) return __uint_as_float(i ? word & 0xFFFF0000u : word << 16);
  else return (float)__builtin_bit_cast(f16_t, (uint16_t)(i ? word >> 16 : word));
}

}  // namespace choco
