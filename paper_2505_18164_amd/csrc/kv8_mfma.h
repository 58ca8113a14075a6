// What the matrix-core kernels of the 8-bit cache share.
#pragma once

#include "kv8_device.h"

namespace mdi {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Two fp32 values as a pair of bf16 by dropping their low halves: exact for codes, which have seven digits.
__device__ __forceinline__ uint32_t high_halves(float lo, float hi) {
  return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}
template <int N> __device__ __forceinline__ float code_of(uint32_t w) { return (float)(int8_t)(w >> (8 * N)); }   // byte N

__device__ __forceinline__ float exp2_raw(float x) { return __builtin_amdgcn_exp2f(x); }

}  // namespace mdi
