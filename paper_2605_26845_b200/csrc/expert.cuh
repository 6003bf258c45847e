// What the expert kernels share: element types, activations, groups of rows.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "common.cuh"

namespace moesched {

// two neighbouring values of a 16-bit type, and single ones, from and to float
template <typename T>
struct Pair;
template <>
struct Pair<__nv_bfloat16> {
  static __device__ __forceinline__ float2 to_float(unsigned v) {
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
  }
  static __device__ __forceinline__ unsigned from_float(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const unsigned*>(&v);
  }
};
template <>
struct Pair<__half> {
  static __device__ __forceinline__ float2 to_float(unsigned v) {
    return __half22float2(*reinterpret_cast<const __half2*>(&v));
  }
  static __device__ __forceinline__ unsigned from_float(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const unsigned*>(&v);
  }
};
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ void put(__nv_bfloat16* to, float v) { *to = __float2bfloat16_rn(v); }
__device__ __forceinline__ void put(__half* to, float v) { *to = __float2half_rn(v); }

// Activation of the gate and its slope. SiLU a s(a), slope s + a s (1 - s), s the logistic function; GELU a F(a), slope
// F + a f(a), F and f the normal distribution and its density.
template <int ACT>
__device__ __forceinline__ float activation(float a) {
  if constexpr (ACT == MOESCHED_ACT_SILU) return __fdividef(a, 1.0f + __expf(-a));
  return 0.5f * a * erfcf(a * -0.70710678118654752f);
}
template <int ACT>
__device__ __forceinline__ void activation_slope(float a, float& value, float& slope) {
  if constexpr (ACT == MOESCHED_ACT_SILU) {
    const float s = __fdividef(1.0f, 1.0f + __expf(-a));
    value = a * s;
    slope = s + value * (1.0f - s);
  } else {
    const float F = 0.5f * erfcf(a * -0.70710678118654752f);
    value = a * F;
    slope = F + a * 0.39894228040143268f * __expf(-0.5f * a * a);
  }
}

// Rows of group g, or none where the offsets are not in order: no offsets make a kernel leave its tensors.
__device__ __forceinline__ int2 rows_of_group(const int32_t* offsets, int g, int R) {
  const int begin = offsets[g], end = offsets[g + 1];
  return begin >= 0 && begin <= end && end <= R ? make_int2(begin, end) : make_int2(0, 0);
}

}  // namespace moesched
