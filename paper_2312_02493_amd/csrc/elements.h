// Element types of the operators around the step: reading them as float32 and rounding back.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace artopk {

enum { kTypeF32 = 0, kTypeBf16 = 1, kTypeF16 = 2 };  // as ARTOPK_G_F32 ..

// Sixteen bytes of elements; whole ones are read and written at 16-byte aligned places only.
template <class T>
struct alignas(16) Vec16 {
  T e[16 / sizeof(T)];
};

// `V` elements at p as float32; V is 1 or what sixteen bytes hold.
template <int V, class T>
__device__ __forceinline__ void load_elems(float (&out)[V], const T* p) {
  if constexpr (V == 1) {
    out[0] = static_cast<float>(*p);
  } else {
    static_assert(V * sizeof(T) == 16, "");
    const Vec16<T> v = *reinterpret_cast<const Vec16<T>*>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = static_cast<float>(v.e[i]);
  }
}

// The same back, each rounded to nearest (ties to even).
template <int V, class T>
__device__ __forceinline__ void store_elems(T* p, const float (&in)[V]) {
  if constexpr (V == 1) {
    *p = static_cast<T>(in[0]);
  } else {
    static_assert(V * sizeof(T) == 16, "");
    Vec16<T> v;
#pragma unroll
    for (int i = 0; i < V; ++i) v.e[i] = static_cast<T>(in[i]);
    *reinterpret_cast<Vec16<T>*>(p) = v;
  }
}

}  // namespace artopk
