// What the kernels on tokens' rows share: vectors of 16 bytes in the types' 32-bit values.
#pragma once

#include "expert.cuh"

namespace moesched {

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ void put(float* to, float v) { *to = v; }

// 16 bytes of type T: COUNT values
template <typename T>
struct Vec {
  static constexpr int COUNT = 16 / sizeof(T);
  static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[COUNT]) {
    const unsigned w[4] = {v.x, v.y, v.z, v.w};
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int q = 0; q < 4; ++q) f[q] = __uint_as_float(w[q]);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if constexpr (std::is_same_v<T, __nv_bfloat16>) {
          f[2 * q] = __uint_as_float(w[q] << 16);
          f[2 * q + 1] = __uint_as_float(w[q] & 0xffff0000u);
        } else {
          const float2 both = __half22float2(*reinterpret_cast<const __half2*>(&w[q]));
          f[2 * q] = both.x;
          f[2 * q + 1] = both.y;
        }
      }
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[COUNT]) {
    if constexpr (sizeof(T) == 4)
      return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    else
      return make_uint4(Pair<T>::from_float(f[0], f[1]), Pair<T>::from_float(f[2], f[3]), Pair<T>::from_float(f[4], f[5]),
                        Pair<T>::from_float(f[6], f[7]));
  }
};

// Tokens and rows pass once: they are not kept in L1. (Not the read-only path: an output may take the place of an input.)
__device__ __forceinline__ uint4 load_once(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ uint2 load_once8(const void* p) {
  uint2 v;
  asm volatile("ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p) : "memory");
  return v;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
  return v;
}

template <typename Kernel, typename... Args>
cudaError_t launch(Kernel kern, long long ctas, int threads, size_t smem, cudaStream_t stream, Args... args) {
  if (cudaError_t e = permit_shared_memory(kern, smem); e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  return cudaLaunchKernelEx(&cfg, kern, args...);
}

// `call` with a value of the type that dtype names, which is one of the three
template <typename Call>
cudaError_t with_type(int dtype, Call call) {
  if (dtype == MOESCHED_BF16) return call(__nv_bfloat16());
  if (dtype == MOESCHED_FP16) return call(__half());
  return call(float());
}

}  // namespace moesched
