// Element access shared by the row-wise kernels: fp32 and bfloat16 storage,
// fp32 arithmetic, nearest-even rounding when a bfloat16 is written.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace sscn {

__device__ __forceinline__ float bf16_bits_f32(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }

// Round to nearest, ties to even; NaN stays NaN.
__device__ __forceinline__ uint16_t f32_bf16_bits(float f) {
  uint32_t u = __float_as_uint(f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return (uint16_t)((u >> 16) | 0x40);
  u += 0x7fffu + ((u >> 16) & 1u);
  return (uint16_t)(u >> 16);
}

// Storage types: float, or uint16_t holding bfloat16 bits.
__device__ __forceinline__ float ld(const float* p) { return *p; }
__device__ __forceinline__ float ld(const uint16_t* p) { return bf16_bits_f32(*p); }
__device__ __forceinline__ void st(float* p, float v) { *p = v; }
__device__ __forceinline__ void st(uint16_t* p, float v) { *p = f32_bf16_bits(v); }

// Two bfloat16 in a word, each to nearest, ties to even; NaN stays NaN.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  typedef __bf16 B2 __attribute__((ext_vector_type(2)));
  typedef float F2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(F2{lo, hi}, B2));
}

}  // namespace sscn
