// What the expert kernels share: element types, activations, groups of rows.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "common.cuh"

namespace moesched {

// two neighbouring values of a 16-bit type from float, and single ones from and to float
template <typename T>
struct Pair;
template <>
struct Pair<__nv_bfloat16> {
  static __device__ __forceinline__ unsigned from_float(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const unsigned*>(&v);
  }
};
template <>
struct Pair<__half> {
  static __device__ __forceinline__ unsigned from_float(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const unsigned*>(&v);
  }
};
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ void put(__nv_bfloat16* to, float v) { *to = __float2bfloat16_rn(v); }
__device__ __forceinline__ void put(__half* to, float v) { *to = __float2half_rn(v); }

// The normal distribution F(a), and e = exp(-a^2 / 2) of its density f = e / sqrt(2 pi). F(-|a|) = e t P(t) with t = 1 / (1 + 0.33 |a|),
// where P is the polynomial of degree 8 whose greatest relative error for |a| <= 14 is least (fitted for this; 5.5e-8, and t P(t)
// evaluated in 32 bits 3.4e-7; beyond 14 e is nothing). F also has the error of e, whose argument is rounded: relatively 4e-7 up to |a| = 1,
// 8e-7 up to 4, 5e-6 at 10, 8e-6 at 13, all of them less than a five-hundredth of bfloat16's half step, a sixtieth of fp16's. With erfcf, and the
// exponential once more, the epilogues bound short contractions: 8 experts, 1024 x 4096, 8192 rows in fp16, forward 217 us, so 188
// (SiLU 175), backward 552 and 528.
__device__ __forceinline__ float normal(float a, float& e) {
  e = __expf(-0.5f * a * a);
  const float t = __fdividef(1.0f, fmaf(0.33f, fabsf(a), 1.0f));
  float p = fmaf(-0.0208072793f, t, 0.123078562f);
  p = fmaf(p, t, -0.267183691f);
  p = fmaf(p, t, 0.22462818f);
  p = fmaf(p, t, -0.0565253757f);
  p = fmaf(p, t, 0.121818744f);
  p = fmaf(p, t, 0.111065961f);
  p = fmaf(p, t, 0.132302776f);
  p = fmaf(p, t, 0.131622165f);
  const float below = e * t * p;
  return a < 0.0f ? below : 1.0f - below;
}

// Activation of the gate and its slope. SiLU a s(a), slope s + a s (1 - s), s the logistic function; GELU a F(a), slope
// F + a f(a), F and f the normal distribution and its density.
template <int ACT>
__device__ __forceinline__ float activation(float a) {
  if constexpr (ACT == MOESCHED_ACT_SILU) return __fdividef(a, 1.0f + __expf(-a));
  float e;
  return a * normal(a, e);
}
template <int ACT>
__device__ __forceinline__ void activation_slope(float a, float& value, float& slope) {
  if constexpr (ACT == MOESCHED_ACT_SILU) {
    const float s = __fdividef(1.0f, 1.0f + __expf(-a));
    value = a * s;
    slope = s + value * (1.0f - s);
  } else {
    float e;
    const float F = normal(a, e);
    value = a * F;
    slope = fmaf(a * 0.39894228040143268f, e, F);
  }
}

// Rows of group g, or none where the offsets are not in order: no offsets make a kernel leave its tensors.
__device__ __forceinline__ bool rows_in_order(int2 span, int R) { return span.x >= 0 && span.x <= span.y && span.y <= R; }
__device__ __forceinline__ int2 rows_of_group(const int32_t* offsets, int g, int R) {
  const int2 span = make_int2(offsets[g], offsets[g + 1]);
  return rows_in_order(span, R) ? span : make_int2(0, 0);
}

// A call that fails leaves NaN in its outputs, so that it shows without its status, which nobody may have asked for. This is one in 32 bits,
// and twice one in either type of 16.
constexpr unsigned NANS = 0x7fff7fffu;
// `value` all over a tensor (16-byte aligned, an even number of bytes): share `part` of `parts`, by all threads of a CTA
static __device__ __noinline__ void fill(void* to, size_t bytes, unsigned value, unsigned part, unsigned parts) {
  const size_t whole = bytes / 16;
  for (size_t q = (size_t)part * blockDim.x + threadIdx.x; q < whole; q += (size_t)parts * blockDim.x)
    static_cast<uint4*>(to)[q] = make_uint4(value, value, value, value);
  if (part == 0 && threadIdx.x < bytes % 16 / 2) static_cast<unsigned short*>(to)[whole * 8 + threadIdx.x] = (unsigned short)value;
}

}  // namespace moesched
