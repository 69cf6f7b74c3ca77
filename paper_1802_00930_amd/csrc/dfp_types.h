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

// N elements as they lie in memory, from p on (aligned to an element only; the vector
// loads of gfx950 take that).  Loaded first and turned into numbers behind all
// loads of a loop: fetch_n is a branch, and what uses the elements in it waits for
// them there (16384 x 8192 BF16 by rows 85.5 us, 72.6 so).
template <int T, int N>
struct __attribute__((packed, aligned(sizeof(typename Elem<T>::type)))) Raw {
  uint32_t w[N * sizeof(typename Elem<T>::type) / 4];
};
// The first `have` of N elements, zero behind them.
template <int T, int N>
__device__ __forceinline__ void fetch_n(const typename Elem<T>::type* p, int64_t have, Raw<T, N>& r) {
  constexpr int E = sizeof(typename Elem<T>::type);
#pragma unroll
  for (int i = 0; i < N * E / 4; ++i) r.w[i] = 0u;
  if (have >= N) {
    r = *reinterpret_cast<const Raw<T, N>*>(p);
  } else if (have > 0) {
#pragma unroll
    for (int i = 0; i < N * E / 4; ++i) {
      if constexpr (E == 4)
        r.w[i] = i < have ? __float_as_uint(p[i]) : 0u;
      else
        r.w[i] = (2 * i < have ? (uint32_t)p[2 * i] : 0u) | (2 * i + 1 < have ? (uint32_t)p[2 * i + 1] << 16 : 0u);
    }
  }
}
template <int T, int N>
__device__ __forceinline__ void up_n(const Raw<T, N>& r, float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if constexpr (sizeof(typename Elem<T>::type) == 4)
      v[i] = __uint_as_float(r.w[i]);
    else
      v[i] = Elem<T>::up((uint16_t)(r.w[i / 2] >> (i % 2 * 16)));
  }
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
template <int T, int N>
__device__ __forceinline__ void load_n(const typename Elem<T>::type* p, int64_t have, float (&v)[N]) {
  Raw<T, N> r;
  fetch_n<T, N>(p, have, r);
  up_n<T, N>(r, v);
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
