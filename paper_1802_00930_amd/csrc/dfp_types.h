// Loads and stores of the element types of the linear layers and weight updates.
#pragma once

#include "dfp_internal.h"

namespace dfp {

template <int T>
struct Elem;
template <>
struct Elem<DFP_F32> {
  typedef float type;
  static __device__ __forceinline__ float up(float v) { return v; }
  static __device__ __forceinline__ float down(float v) { return v; }
};
template <>
struct Elem<DFP_BF16> {
  typedef uint16_t type;
  static __device__ __forceinline__ float up(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
  static __device__ __forceinline__ uint16_t down(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
};
template <>
struct Elem<DFP_F16> {
  typedef uint16_t type;
  static __device__ __forceinline__ float up(uint16_t v) { return (float)__builtin_bit_cast(_Float16, v); }
  static __device__ __forceinline__ uint16_t down(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
};

inline int64_t type_bytes(int32_t type) { return type == DFP_F32 ? 4 : 2; }

// N elements from p (aligned to an element only; the vector loads of gfx950 take that).
template <int T, int N>
__device__ __forceinline__ void load_n(const typename Elem<T>::type* p, float (&v)[N]) {
  typedef typename Elem<T>::type E;
  struct __attribute__((packed, aligned(sizeof(E)))) Raw {
    E e[N];
  };
  const Raw r = *reinterpret_cast<const Raw*>(p);
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = Elem<T>::up(r.e[i]);
}
template <int T, int N>
__device__ __forceinline__ void store_n(typename Elem<T>::type* p, const float (&v)[N]) {
  typedef typename Elem<T>::type E;
  struct __attribute__((packed, aligned(sizeof(E)))) Raw {
    E e[N];
  } r;
#pragma unroll
  for (int i = 0; i < N; ++i) r.e[i] = Elem<T>::down(v[i]);
  *reinterpret_cast<Raw*>(p) = r;
}
// The first `have` of N elements, zero behind them.
template <int T, int N>
__device__ __forceinline__ void load_n(const typename Elem<T>::type* p, int64_t have, float (&v)[N]) {
  if (have >= N) return load_n<T, N>(p, v);
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = i < have ? Elem<T>::up(p[i]) : 0.f;
}
template <int T, int N>
__device__ __forceinline__ void store_n(typename Elem<T>::type* p, int64_t have, const float (&v)[N]) {
  if (have >= N) return store_n<T, N>(p, v);
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (i < have) p[i] = Elem<T>::down(v[i]);
}

// f(integral_constant of the type), for a checked type.
template <class F>
dfp_status with_type(int32_t type, F f) {
  switch (type) {
    case DFP_F32: return f(std::integral_constant<int, DFP_F32>());
    case DFP_BF16: return f(std::integral_constant<int, DFP_BF16>());
    default: return f(std::integral_constant<int, DFP_F16>());
  }
}

}  // namespace dfp
