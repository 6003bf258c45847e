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

// Two products and sums of 32 bits in one instruction; pairs of values as `unpack` leaves them side by side
struct Two {
  unsigned long long v;
};
__device__ __forceinline__ Two two(float lo, float hi) {
  Two t;
  asm("mov.b64 %0, {%1, %2};" : "=l"(t.v) : "f"(lo), "f"(hi));
  return t;
}
__device__ __forceinline__ float2 apart_of(Two t) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(t.v));
  return f;
}
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
  Two d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return d;
}
__device__ __forceinline__ Two mul2(Two a, Two b) {
  Two d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v));
  return d;
}
template <typename T>
__device__ __forceinline__ void pairs_of(const uint4& v, Two (&p)[Vec<T>::COUNT / 2]) {
  float f[Vec<T>::COUNT];
  Vec<T>::unpack(v, f);
#pragma unroll
  for (int e = 0; e < Vec<T>::COUNT / 2; ++e) p[e] = two(f[2 * e], f[2 * e + 1]);
}

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
__device__ __forceinline__ unsigned load_once4(const void* p) {
  unsigned v;
  asm volatile("ld.global.L1::no_allocate.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}

// To shared memory behind the thread's back: read again by the thread that asked for it, after it has waited, so that no barrier is needed.
__device__ __forceinline__ void copy_behind(void* shared, const void* global) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_addr(shared)), "l"(global) : "memory");
}
__device__ __forceinline__ void copies_asked() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LATER>
__device__ __forceinline__ void copies_here() { asm volatile("cp.async.wait_group %0;" ::"n"(LATER) : "memory"); }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
  return v;
}

// early: may be started before the kernel before it, of the same call, is over
template <typename Kernel, typename... Args>
cudaError_t launch(Kernel kern, dim3 ctas, dim3 threads, size_t smem, bool early, cudaStream_t stream, Args... args) {
  if (cudaError_t e = permit_shared_memory(kern, smem); e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = ctas;
  cfg.blockDim = threads;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr = start_early();
  cfg.attrs = &attr;
  cfg.numAttrs = early ? 1 : 0;
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
