// Numbers of 8 bits under a scale: a value x is held as round(x / s), s a power of two, so that the quotient is exact and the rounding to 8 bits the only one.
#pragma once
#include "common.hpp"

namespace mqa {

// e4m3: finite numbers up to 448 = 1.75 2^8, rounded to the nearest, of two the even one; NaN.  int8: -127 .. 127.
template <bool E4M3> struct Held;
template <> struct Held<true> {
  static constexpr uint32_t kMantissa = 0x600000u;      // of the largest number
  static constexpr int kExponent = 8;
  static constexpr float kLargest = 448.f;
};
template <> struct Held<false> {
  static constexpr uint32_t kMantissa = 0x7e0000u;      // 127 = 1.984375 2^6
  static constexpr int kExponent = 6;
  static constexpr float kLargest = 127.f;
};

// The smallest power of two, 2^-126 at least, times the type's largest number is no less than `a` (finite, not negative): a's exponent, one more where its
// mantissa is past the largest number's, less that one's.
template <bool E4M3>
__device__ __forceinline__ float scale_of(float a) {
  const int e = (int)((__float_as_uint(a) + (0x7fffffu - Held<E4M3>::kMantissa)) >> 23) - Held<E4M3>::kExponent;
  return __uint_as_float((uint32_t)max(e, 1) << 23);
}
// 1 / s of a power of two from 2^-126 to 2^126.
__device__ __forceinline__ float inverse_of(float s) { return __uint_as_float(0x7f000000u - __float_as_uint(s)); }

// Four quotients in 8 bits each.  What is too large (an infinity) becomes the largest number; NaN is e4m3's NaN, int8's 0.
template <bool E4M3>
__device__ __forceinline__ uint32_t round4(const float4& x) {
  constexpr float top = Held<E4M3>::kLargest;
  auto within = [](float y) { return y != y ? (E4M3 ? y : 0.f) : fminf(fmaxf(y, -top), top); };
  const float a = within(x.x), b = within(x.y), c = within(x.z), d = within(x.w);
  if constexpr (E4M3) {
    int u = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, u, true);
  } else {
    return ((uint32_t)(int)rintf(a) & 0xffu) | ((uint32_t)(int)rintf(b) & 0xffu) << 8 | ((uint32_t)(int)rintf(c) & 0xffu) << 16 | (uint32_t)(int)rintf(d) << 24;
  }
}
template <bool E4M3>
__device__ __forceinline__ float4 values4(uint32_t u) {
  if constexpr (E4M3) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(u, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(u, true);
    return make_float4(lo[0], lo[1], hi[0], hi[1]);
  } else {
    return make_float4((int8_t)u, (int8_t)(u >> 8), (int8_t)(u >> 16), (int8_t)(u >> 24));
  }
}

}  // namespace mqa
