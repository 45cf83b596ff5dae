// Loads and stores of float, bfloat16 and half vectors as 32-bit floats.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gba.h"

namespace gba {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// V elements of type T at any element-aligned address: one access of up to 16
// bytes where the vector has as many (rows of odd widths and strides begin at
// such addresses, and the hardware takes them).
template <typename T, int V>
struct VecOf {
  typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T))));
};

// 16 bytes of T
template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);

template <typename T, int V>
__device__ __forceinline__ void load_vec(const T* __restrict__ p, float (&o)[V]) {
  const typename VecOf<T, V>::type v = *reinterpret_cast<const typename VecOf<T, V>::type*>(p);
#pragma unroll
  for (int e = 0; e < V; ++e) o[e] = (float)v[e];
}
// the first `count` (1 to V) of them, the rest 0
template <typename T, int V>
__device__ __forceinline__ void load_part(const T* __restrict__ p, int count, float (&o)[V]) {
  if (count >= V) {
    load_vec<T, V>(p, o);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) o[e] = e < count ? (float)p[e] : 0.0f;
  }
}
// rounded to T once, to the nearest (ties to even); PAST: past the caches
template <typename T, int V, bool PAST = false>
__device__ __forceinline__ void store_vec(T* __restrict__ p, const float (&o)[V]) {
  typedef typename VecOf<T, V>::type vec;
  vec v;
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = (T)o[e];
  if constexpr (PAST) __builtin_nontemporal_store(v, reinterpret_cast<vec*>(p));
  else *reinterpret_cast<vec*>(p) = v;
}
template <typename T, int V, bool PAST = false>
__device__ __forceinline__ void store_part(T* __restrict__ p, int count, const float (&o)[V]) {
  if (count >= V) {
    store_vec<T, V, PAST>(p, o);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (e < count) p[e] = (T)o[e];
  }
}

// The same with the type in a (uniform) value.
template <int V>
__device__ __forceinline__ void load_part(const void* __restrict__ p, int type, int64_t at, int count, float (&o)[V]) {
  if (type == GBA_F32) load_part<float, V>(static_cast<const float*>(p) + at, count, o);
  else if (type == GBA_BF16) load_part<bf16_t, V>(static_cast<const bf16_t*>(p) + at, count, o);
  else load_part<f16_t, V>(static_cast<const f16_t*>(p) + at, count, o);
}
template <int V>
__device__ __forceinline__ void store_part(void* __restrict__ p, int type, int64_t at, int count, const float (&o)[V]) {
  if (type == GBA_F32) store_part<float, V>(static_cast<float*>(p) + at, count, o);
  else if (type == GBA_BF16) store_part<bf16_t, V>(static_cast<bf16_t*>(p) + at, count, o);
  else store_part<f16_t, V>(static_cast<f16_t*>(p) + at, count, o);
}

}  // namespace gba
