// e4m3 values (1 sign, 4 exponent, 3 fraction bits; largest 448, no infinity) as the kernels of the 8-bit cache take them.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "ds_common.cuh"

namespace ds {

// Two values, the first in the low byte; rounded to the nearest, ties to even; NaN stays NaN.
__device__ __forceinline__ uint32_t pack_e4m3(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t pack_e4m3x4(float a, float b, float c, float d) {
  return pack_e4m3(a, b) | (pack_e4m3(c, d) << 16);
}
// The low or high two bytes of a word as two fp16 values, which hold every e4m3 value.
__device__ __forceinline__ uint32_t halves_lo(uint32_t w) {
  uint32_t r;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\t}" : "=r"(r) : "r"(w));
  return r;
}
__device__ __forceinline__ uint32_t halves_hi(uint32_t w) {
  uint32_t r;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, h;\n\t}" : "=r"(r) : "r"(w));
  return r;
}
__device__ __forceinline__ float2 halves_f32(uint32_t h) { return __half22float2(*reinterpret_cast<const __half2 *>(&h)); }

// The product cut off at 24 bits, its last bit set if that lost something: rounding it to two bits fewer or less gives the product
// rounded once.  The product must be 2^-100 or more in magnitude, or zero; what passes the largest value becomes that value.
__device__ __forceinline__ float mul_to_odd(float a, float b) {
  const float r = __fmul_rz(a, b), rest = fmaf(a, b, -r);
  return rest > 0.f || rest < 0.f ? __uint_as_float(__float_as_uint(r) | 1u) : r;
}

// Whether one of a word's four bytes is NaN.
__device__ __forceinline__ bool any_nan_e4m3(uint32_t w) { return __vcmpeq4(w & 0x7f7f7f7fu, 0x7f7f7f7fu) != 0; }

}  // namespace ds
