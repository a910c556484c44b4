// Rows of K and V into 8-bit codes and scales: what the kernels that write the cache share.
#pragma once

#include <stdint.h>

namespace fastav {

// The largest magnitude of eight bf16 values, twice; what is not a number is larger than everything else.
__device__ __forceinline__ unsigned larger(unsigned a, unsigned b) {
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(a), "r"(b));
  return a;
}
__device__ __forceinline__ unsigned magnitudes(unsigned a) {
  asm("abs.bf16x2 %0, %0;" : "+r"(a));
  return a;
}
__device__ __forceinline__ unsigned top_of(const uint4& x) { return larger(larger(magnitudes(x.x), magnitudes(x.y)), larger(magnitudes(x.z), magnitudes(x.w))); }

// code_i = round(x_i L / top) to nearest, ties to even, exactly.  x_i L has at most 15 bits, so it is exact in fp32, and the quotient of a
// 15-bit and an 8-bit number that is no tie is at least 2^-16 of itself away from one.  Everything is scaled by a power of two that brings
// `top` near 1 (and leaves room for L), so that nothing overflows and 1 / top is normal.
//
// An approximate quotient corrected once by its remainder (q + (n - q t) / t: an ulp off at most, and exact where the quotient is short)
// rounds as the true one does.
struct Quotient {
  float2 to, less, r;  // L times the power of two; -top times it; the reciprocal of that
  __device__ Quotient(unsigned top, float largest) {
    const int e = (int)(top >> 7);
    const float power = __uint_as_float((unsigned)min(max(254 - e, 1), 240) << 23), t = top ? __uint_as_float(top << 16) * power : 1.f, inv = __fdividef(1.f, t);
    to = make_float2(power * largest, power * largest);
    less = make_float2(-t, -t);
    r = make_float2(inv, inv);
  }
  __device__ float2 operator()(const float2& two) const {
    const float2 n = __fmul2_rn(two, to), q = __fmul2_rn(n, r);
    return __ffma2_rn(__ffma2_rn(q, less, n), r, q);
  }
};
// int8, in one step: x times L / top rounded UP.  A quotient that is no tie is not moved across one.  A tie, 254 x = (2 k + 1) top, needs 127
// to divide 2 k + 1 or top's eight bits: then it is 63.5, which goes up to 64, or top is 254 times a power of two and 127 / top and
// every product are exact.  So one fused multiply-add with 1.5 * 2^23 leaves the code in the sum's low bits.  (Not where L / top is too large.)
constexpr unsigned kLeastTop = 0x1000;  // 2^-95
__device__ __forceinline__ float inverse_up(unsigned top) {
  const int e = (int)(top >> 7);
  const float power = __uint_as_float((unsigned)max(254 - e, 1) << 23), t = __uint_as_float(top << 16) * power, inv = __fdividef(1.f, t);
  float x = 127.f * inv;
  x = fmaf(fmaf(-x, t, 127.f), inv, x);                                           // within an ulp
  const float below = __uint_as_float(__float_as_uint(x) - 1);
  if (fmaf(-x, t, 127.f) > 0.f) x = __uint_as_float(__float_as_uint(x) + 1);      // (the remainders are exact)
  else if (fmaf(-below, t, 127.f) <= 0.f) x = below;
  return x * power;
}
// top / L, to nearest: a quotient within an ulp, corrected by its exact remainder times the nearest reciprocal (Markstein), where the remainder is normal.
template <bool FP8>
__device__ __forceinline__ float scale_of(unsigned top) {
  constexpr float kLargest = FP8 ? 448.f : 127.f, kInverse = 1.f / kLargest;
  const float t = __uint_as_float(top << 16);
  if (top < kLeastTop) return __fdiv_rn(t, kLargest);
  const float q = t * kInverse;
  return fmaf(fmaf(-q, kLargest, t), kInverse, q);
}

__device__ __forceinline__ unsigned low_bytes(const float2& a, const float2& b) {
  return __byte_perm(__byte_perm(__float_as_uint(a.x), __float_as_uint(a.y), 0x0040), __byte_perm(__float_as_uint(b.x), __float_as_uint(b.y), 0x0040), 0x5410);
}
__device__ __forceinline__ unsigned pack_e4m3(const float2& a, const float2& b) {
  unsigned short lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(a.y), "f"(a.x));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(b.y), "f"(b.x));
  return (unsigned)lo | (unsigned)hi << 16;
}

__device__ __forceinline__ unsigned two_bf16(float lo, float hi) {
  unsigned r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float2 both(unsigned two) { return make_float2(__uint_as_float(two << 16), __uint_as_float(two & 0xFFFF0000u)); }
template <bool FP8>
__device__ __forceinline__ uint2 quantise8(const uint4& x, unsigned top) {
  if (FP8) {
    const Quotient q(top, 448.f);
    return make_uint2(pack_e4m3(q(both(x.x)), q(both(x.y))), pack_e4m3(q(both(x.z)), q(both(x.w))));
  }
  const float2 round = make_float2(12582912.f, 12582912.f);
  if (top < kLeastTop) {
    const Quotient q(top, 127.f);
    return make_uint2(low_bytes(__fadd2_rn(q(both(x.x)), round), __fadd2_rn(q(both(x.y)), round)), low_bytes(__fadd2_rn(q(both(x.z)), round), __fadd2_rn(q(both(x.w)), round)));
  }
  const float up = inverse_up(top);
  const float2 r = make_float2(up, up);
  return make_uint2(low_bytes(__ffma2_rn(both(x.x), r, round), __ffma2_rn(both(x.y), r, round)), low_bytes(__ffma2_rn(both(x.z), r, round), __ffma2_rn(both(x.w), r, round)));
}

}  // namespace fastav
