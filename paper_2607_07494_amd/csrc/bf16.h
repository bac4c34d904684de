// bfloat16 by its bits: a float32's upper half.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gift {

// the lower and the upper one of a word
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// float32 -> bfloat16, to nearest even; a NaN stays one
__device__ __forceinline__ uint32_t to_bf16(float x) {
  const uint32_t u = __float_as_uint(x);
  return x != x ? (u >> 16 | 0x40u) : (u + 0x7fffu + (u >> 16 & 1u)) >> 16;
}

}  // namespace gift
