// Device helpers of the products with 4-bit codes.
#pragma once
#include "common.h"

namespace akvs {

typedef __attribute__((ext_vector_type(2))) int i32x2_t;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2_t;

// (w & mask) | bits in one instruction. It takes one operand from a scalar register, and no constant:
// written with constants the compiler makes two of it (the other constant in a vector register for
// good is what this costs).
struct CodeBits {
  uint32_t mask, bits;
};
__device__ __forceinline__ CodeBits code_bits(uint32_t mask, uint32_t bits) {
  CodeBits x;
  asm("s_mov_b32 %0, %1" : "=s"(x.mask) : "i"(mask));
  asm("v_mov_b32 %0, %1" : "=v"(x.bits) : "i"(bits));
  return x;
}
__device__ __forceinline__ uint32_t and_or(uint32_t w, CodeBits c) { return (w & c.mask) | c.bits; }

// Eight codes as bf16 16 + c, in the order 0, 4, 1, 5, 2, 6, 3, 7; c: bf16_bits().
__device__ __forceinline__ CodeBits bf16_bits() { return code_bits(0x00780078u, 0x41804180u); }
__device__ __forceinline__ bf16x8_t codes8(uint32_t w, CodeBits c) {
  const u32x4_t x = {and_or(w << 3, c), and_or(w >> 1, c), and_or(w >> 5, c), and_or(w >> 9, c)};
  return __builtin_bit_cast(bf16x8_t, x);
}
// Two fp16, rounded to nearest even.
__device__ __forceinline__ uint32_t pack_half2(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t){a, b}, f16x2_t));
}
// Eight bf16 in that order.
__device__ __forceinline__ bf16x8_t order8(u32x4_t q) {
  const u32x4_t x = {(q[0] & 0xffffu) | (q[2] << 16), (q[0] >> 16) | (q[2] & 0xffff0000u),
                     (q[1] & 0xffffu) | (q[3] << 16), (q[1] >> 16) | (q[3] & 0xffff0000u)};
  return __builtin_bit_cast(bf16x8_t, x);
}
__device__ __forceinline__ float scale_of(uint32_t m) {
  return (float)__builtin_bit_cast(f16x2_t, m)[0];
}
// |scale| as the fp16 it is, whose order is that of the integers; 0 where it is not finite.
__device__ __forceinline__ uint32_t scale_bits(uint32_t m) {
  const uint32_t x = m & 0x7fffu;
  return x < 0x7c00u ? x : 0u;
}
__device__ __forceinline__ float zero_of(uint32_t m) {
  return (float)__builtin_bit_cast(f16x2_t, m)[1];
}

// Whether scale * code + zero may lie past fp16's range, or is no number: true at |scale| > 2^11 or
// |zero| > 2^15 (fp16 in the order of integers, both at once).
__device__ __forceinline__ bool wide_values(uint32_t m) {
  return (((m & 0x7fff7fffu) + 0x07ff17ffu) & 0x80008000u) != 0;
}

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8_t;
// 1024 + c and 1024 + 16 c are fp16 numbers whose low bits are the nibble where it lies.
struct F16Bits {
  CodeBits lo, hi;
};
__device__ __forceinline__ F16Bits f16_bits() {
  F16Bits x{code_bits(0x000f000fu, 0x64006400u), code_bits(0x00f000f0u, 0x64006400u)};
  x.hi.bits = x.lo.bits;
  return x;
}
// Eight codes as fp16 1024 + c (nibbles 0, 4, 2, 6) and 1024 + 16 c (1, 5, 3, 7), in that order of
// pairs: 0, 4, 1, 5, 2, 6, 3, 7.
__device__ __forceinline__ f16x8_t raw8(uint32_t w, F16Bits b) {
  const u32x4_t x = {and_or(w, b.lo), and_or(w, b.hi), and_or(w >> 8, b.lo), and_or(w >> 8, b.hi)};
  return __builtin_bit_cast(f16x8_t, x);
}
// Eight codes as fp16, exactly, in that order.
__device__ __forceinline__ f16x8_t exact8(uint32_t w, F16Bits b) {
  const f16x2_t down = {(_Float16)-1024.f, (_Float16)-1024.f};
  const f16x2_t part = {(_Float16)0.0625f, (_Float16)0.0625f};
  const f16x2_t off = {(_Float16)-64.f, (_Float16)-64.f};
  union {
    f16x2_t h[4];
    f16x8_t v;
  } x;
  x.v = raw8(w, b);
#pragma unroll
  for (int i = 0; i < 4; i += 2) {
    x.h[i] = x.h[i] + down;
    x.h[i + 1] = __builtin_elementwise_fma(x.h[i + 1], part, off);
  }
  return x.v;
}
// scale * code + zero in fp16, rounded once.
__device__ __forceinline__ f16x8_t values8(uint32_t w, f16x2_t scale, f16x2_t zero, F16Bits b) {
  union {
    f16x2_t h[4];
    f16x8_t v;
  } x;
  x.v = exact8(w, b);
#pragma unroll
  for (int i = 0; i < 4; ++i) x.h[i] = __builtin_elementwise_fma(x.h[i], scale, zero);
  return x.v;
}
// The upper half of the wave's a against the lower half of its b.
__device__ __forceinline__ void swap_halves(uint32_t &a, uint32_t &b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}
// o[j]: what lane l % 16 of the wave's j-th 16 lanes has, in all lanes.
__device__ __forceinline__ void spread4(uint32_t v, uint32_t (&o)[4]) {
  const auto h = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  const auto a = __builtin_amdgcn_permlane16_swap(h[0], h[0], false, false);
  const auto b = __builtin_amdgcn_permlane16_swap(h[1], h[1], false, false);
  o[0] = a[0];
  o[1] = a[1];
  o[2] = b[0];
  o[3] = b[1];
}

}  // namespace akvs
