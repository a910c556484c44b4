// 8-bit codes as operands of mma.sync in f16.  int8 codes and e4m3 values are exact in f16.
#pragma once

#include <stdint.h>

namespace fastav {

// Four codes -> two pairs of f16 (bytes 0 and 1; bytes 2 and 3).  int8: the code plus 128 as the low bits of an f16 in [1024, 2048), less 1152.
template <bool FP8>
__device__ __forceinline__ void four_codes(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if (FP8) {
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(w));
  } else {
    w ^= 0x80808080u;
    const uint32_t magic = 0x64646464u, less = 0xE480E480u;  // -1152, twice
    asm("add.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(__byte_perm(w, magic, 0x4140)), "r"(less));
    asm("add.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(__byte_perm(w, magic, 0x4342)), "r"(less));
  }
}

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t two_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t pair_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// The power of two that brings a magnitude with these float bits into [1, 2) (into f32's range where it is tiny or huge; 1 where it is not finite).
__device__ __forceinline__ float to_one(float magnitude) {
  const int e = (int)(__float_as_uint(magnitude) >> 23 & 255u);
  return e == 255 ? 1.f : __uint_as_float((unsigned)min(max(254 - e, 1), 240) << 23);  // (room for a further factor)
}

// 1 / x of a power of two that to_one gives (times a small one).
__device__ __forceinline__ float inverse_power(float x) { return __uint_as_float((254u << 23) - __float_as_uint(x)); }

// m + log2(l), -inf for l = 0.  m and log2(l) may be large where their sum is not (m holds the exponents of values' scales), so l's exponent goes to m
// first, exactly: 70 + log2f(2^-70) alone is off by 2^-18.
__device__ __forceinline__ float plus_log2(float m, float l) {
  if (l == 0.f) return -INFINITY;
  if (!(l < INFINITY)) return l;
  const int bits = (int)__float_as_uint(l), k = (bits >> 23) - 127;
  return m + (float)k + log2f(__uint_as_float((unsigned)(bits - (k << 23))));
}

// A query row as f16.  It is multiplied by a power of two that lays its largest magnitude on 2^15 .. 2^16 (bf16's largest mantissa there is
// 65,280; f16 ends at 65,504).  Elements of 2^-32 of the largest and more are exact then; f16's last step being 2^-24, smaller ones are off by at
// most 2^-40 of it.  (Laid on 1 .. 2, those below 2^-17 lost bits, and that showed wherever no key answers the largest element.)
//
// A logit is (sum of query and code) * (the key's scale 2^-kLogitBits) * (softmax scale 2^kLogitBits / the power of two): the first two factors stay
// below 2^127 for every scale that a bf16 row can have.
constexpr int kQueryBits = 15, kLogitBits = 24;
constexpr float kKeyScaleFactor = 1.f / (1 << kLogitBits);

// ... that power of two, for the largest magnitude's bf16 bits (1 where it is 0 or not finite).
__device__ __forceinline__ float query_power(unsigned top) {
  const int e = (int)(top >> 7);
  return top == 0 || e == 255 ? 1.f : __uint_as_float((unsigned)min(254 + kQueryBits - e, 253) << 23);
}
// ... and what takes it back, times the softmax scale (base 2): never 0, or a hidden key's -inf times it would not be -inf.
__device__ __forceinline__ float query_scale(float scale_log2, float power) {
  const int e = 254 + kLogitBits - (int)(__float_as_uint(power) >> 23);
  return fmaxf(scale_log2 * __uint_as_float((unsigned)min(e, 254) << 23), 1.4e-45f);
}

}  // namespace fastav
