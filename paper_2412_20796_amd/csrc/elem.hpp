// Element types of the operators (chgnet_ops.h): fp32 arithmetic on values held
// in fp32, bf16 or fp16, rounded once where they are stored.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "chgnet_ops.h"

namespace chg {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// V consecutive values (V = 1, 4 or 8), aligned to their total size, at most 16 bytes
template <int V, class T>
__device__ __forceinline__ void load_v(const T* p, float (&v)[V]) {
  if constexpr (V * sizeof(T) > 16) {
    float a[V / 2], b[V / 2];
    load_v<V / 2>(p, a);
    load_v<V / 2>(p + V / 2, b);
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = k < V / 2 ? a[k % (V / 2)] : b[k % (V / 2)];
  } else {
    typedef T vec __attribute__((ext_vector_type(V)));
    const vec t = *reinterpret_cast<const vec*>(p);
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = (float)t[k];
  }
}
template <int V, class T>
__device__ __forceinline__ void store_v(T* p, const float (&v)[V]) {
  if constexpr (V * sizeof(T) > 16) {
    float a[V / 2], b[V / 2];
#pragma unroll
    for (int k = 0; k < V / 2; ++k) {
      a[k] = v[k];
      b[k] = v[V / 2 + k];
    }
    store_v<V / 2>(p, a);
    store_v<V / 2>(p + V / 2, b);
  } else {
    typedef T vec __attribute__((ext_vector_type(V)));
    vec t;
#pragma unroll
    for (int k = 0; k < V; ++k) t[k] = (T)v[k];
    *reinterpret_cast<vec*>(p) = t;
  }
}

// The same past the caches (nontemporal), for values that are read once and
// results that others than this kernel read.
template <int V, class T>
__device__ __forceinline__ void load_nt(const T* p, float (&v)[V]) {
  static_assert(V * sizeof(T) <= 16, "one access");
  typedef T vec __attribute__((ext_vector_type(V)));
  const vec t = __builtin_nontemporal_load(reinterpret_cast<const vec*>(p));
#pragma unroll
  for (int k = 0; k < V; ++k) v[k] = (float)t[k];
}
template <int V, class T>
__device__ __forceinline__ void store_nt(T* p, const float (&v)[V]) {
  static_assert(V * sizeof(T) <= 16, "one access");
  typedef T vec __attribute__((ext_vector_type(V)));
  vec t;
#pragma unroll
  for (int k = 0; k < V; ++k) t[k] = (T)v[k];
  __builtin_nontemporal_store(t, reinterpret_cast<vec*>(p));
}

// Input bytes of a call from which it loads them past the caches: half of the
// last cache's 256 MB (by layouts that have such loads: see there). (The gate: 154 MB of z after the product that wrote it: 121 -> 115
// us with what comes before and after; 87 MB: the same; 44 MB that no kernel
// has touched lately: 33 -> 40.)
constexpr int64_t kFarBytes = 128 << 20;

inline int elem_size(int32_t dtype) { return dtype == CHGNET_F32 ? 4 : dtype == CHGNET_BF16 || dtype == CHGNET_F16 ? 2 : 0; }
// calls f with a value of the (valid) type
template <class F>
int with_type(int32_t dtype, F&& f) {
  if (dtype == CHGNET_F32) return f(float{});
  if (dtype == CHGNET_BF16) return f(bf16_t{});
  return f(f16_t{});
}
inline bool aligned_to(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

}  // namespace chg
