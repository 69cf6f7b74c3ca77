// Scale of a row and rounding of its elements to INT8 (see dfp.h).
#pragma once

#include <type_traits>

#include "dfp_internal.h"
#include "dfp_round.h"

#pragma clang fp contract(off)

namespace dfp {

// Scale of a maximum (FP32 bits, NaN and Inf above every finite one): s as
// stored, and the pair (s, x) is multiplied by `up` before the division so that a
// subnormal s has all its bits in the reciprocal.
struct I8Scale {
  float s, su, inv, up;
  bool live;
};
// Scale s with the reciprocal that i8_scale found for it (0: the row's integers are 0).
__device__ __forceinline__ I8Scale i8_scale_of(float s, float inv) {
  I8Scale r;
  r.s = s;
  r.live = inv != 0.f;
  r.up = s < 0x1p-60f ? 0x1p64f : 1.f;
  r.su = s * r.up;
  r.inv = inv;
  return r;
}
__device__ __forceinline__ I8Scale i8_scale(uint32_t amax_bits) {
  const bool finite = amax_bits < 0x7f800000u;
  const float s = finite ? __uint_as_float(amax_bits) / 127.f : __uint_as_float(0x7fc00000u);
  I8Scale r = i8_scale_of(s, 0.f);
  r.live = finite && s > 0.f;
  r.inv = r.live ? 1.f / r.su : 0.f;
  return r;
}

// round(x / s).  x * inv is within one integer of it, and e = x - q s is exact:
// x and q s are multiples of the ulp of the smaller of x and s, and |e| <= s.
template <int MODE>
__device__ __forceinline__ int32_t i8_round(float x, const I8Scale& k, uint32_t u) {
  const float xu = x * k.up;
  float q = rintf(xu * k.inv);
  float e = fmaf(-q, k.su, xu);
  const float h = 2.f * fabsf(e);
  const bool move = h > k.su || (h == k.su && ((int32_t)q & 1));
  const float step = move ? copysignf(1.f, e) : 0.f;
  q += step;
  if (MODE == DFP_ROUND_STOCHASTIC) {
    e = fmaf(-step, k.su, e);
    const int64_t R = (int64_t)floor((double)(e / k.su) * 0x1p32);
    q += (float)((int32_t)(R >> 32) + (u < (uint32_t)R ? 1 : 0));
  }
  return (int32_t)fminf(fmaxf(q, -127.f), 127.f);
}

// The low bytes of four words.
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u),
                               0x05040100u);
}

// Philox words of N consecutive flat indices.
template <int N>
__device__ __forceinline__ void words(uint64_t idx, uint32_t k0, uint32_t k1, uint32_t role, uint32_t (&u)[N]) {
  uint64_t at = ~0ull;
  uint4 w = make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint64_t q = (idx + i) >> 2;
    if (q != at) {
      at = q;
      w = philox4x32_10(make_uint4((uint32_t)q, (uint32_t)(q >> 32), role, 0u), k0, k1);
    }
    const uint32_t s = (uint32_t)(idx + i) & 3;
    u[i] = s == 0 ? w.x : s == 1 ? w.y : s == 2 ? w.z : w.w;
  }
}

// The nearest integers of eight elements with scales k[i] (or one for all, k[0]), two
// bytes' worth of answers at a time in the common case: r = x inv + 1.5 2^23 rounds x inv to
// an integer and holds it in its low byte.  x inv is off from x / s by at most 127
// 2^-23, so the integer is right unless it is that near to a tie, d = 1/2; then, and
// for subnormal scales, the exact rounding above.  Memory's rate leaves about 20
// operations an element: the exact rounding alone takes them all (16384 x 8192 BF16
// 108 us by it).
template <bool EACH>
__device__ __forceinline__ bool i8_nearest8(const float (&v)[8], const I8Scale* k, uint32_t (&o)[8]) {
  float far = 0.f;
  bool plain = true;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const I8Scale& s = k[EACH ? i : 0];
    const float r = fmaf(v[i], s.inv, 12582912.f), d = fmaf(v[i], s.inv, 12582912.f - r);
    far = fmaxf(far, fabsf(d));
    if (EACH || i == 0) plain = plain && s.up == 1.f;
    o[i] = __float_as_uint(r);
  }
  return plain && far < 0.49998f;
}

template <int MODE>
__device__ __forceinline__ uint2 i8_round8(const float (&v)[8], const I8Scale& k, uint64_t idx, uint32_t k0,
                                           uint32_t k1, uint32_t role) {
  uint32_t q[8];
  if (MODE != DFP_ROUND_NEAREST || !i8_nearest8<false>(v, &k, q)) {
    uint32_t u[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (MODE == DFP_ROUND_STOCHASTIC) words<8>(idx, k0, k1, role, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = (uint32_t)i8_round<MODE>(v[i], k, u[i]);
  }
  const uint2 o = make_uint2(low_bytes(q[0], q[1], q[2], q[3]), low_bytes(q[4], q[5], q[6], q[7]));
  return k.live ? o : make_uint2(0, 0);
}

// f(integral_constant of the rounding), for a checked rounding.
template <class F>
dfp_status with_mode(int32_t rounding, F f) {
  if (rounding == DFP_ROUND_STOCHASTIC) return f(std::integral_constant<int, DFP_ROUND_STOCHASTIC>());
  return f(std::integral_constant<int, DFP_ROUND_NEAREST>());
}

}  // namespace dfp
