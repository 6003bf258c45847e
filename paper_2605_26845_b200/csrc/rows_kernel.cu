// Tokens to the rows of the send buffer and back: rows[slot[t k + j]] = x[t], and y[t] = sum_j w_tj rows[slot[t k + j]].
//
// A choice whose slot is not one of the source's T k rows was not sent: it writes nothing and adds nothing. Everything is done token by token, so
// that a token's row is read once for all of its choices, sums are in the order of the choices, and nothing needs the inverse of `slot`.
// One warp has a stretch of a token's row. Memory bounds all of it.
#include <cuda_fp8.h>

#include "token.cuh"

namespace moesched {

constexpr int ROWS_WARPS = 8;      // of a CTA
constexpr int ROWS_AHEAD = 4;      // vectors of a row in flight per lane

// Row of the choice in its source's buffer of `rows` rows, counted from the first source; negative: not sent
__device__ __forceinline__ long long row_of(const int32_t* slot, long long choice, long long source, int rows) {
  const int at = slot[choice];
  return (unsigned)at < (unsigned)rows ? source * rows + at : -1;
}

template <typename V>
__device__ __forceinline__ V load_vec(const void* p) {
  if constexpr (sizeof(V) == 16) return load_once(p);
  else return load_once8(p);
}

template <typename V>
__global__ void __launch_bounds__(32 * ROWS_WARPS) scatter_kernel(long long tokens, int T, int k, int vectors, int parts, int scales,
                                                                  const V* __restrict__ x, const float* __restrict__ scale,
                                                                  const int32_t* __restrict__ slot, V* __restrict__ rows,
                                                                  float* __restrict__ row_scale) {
  const int lane = threadIdx.x & 31;
  const long long item = (long long)blockIdx.x * ROWS_WARPS + (threadIdx.x >> 5), token = item / parts;
  if (token >= tokens) return;
  const int part = (int)(item % parts);
  const long long row = lane < k ? row_of(slot, token * k + lane, token / T, T * k) : -1;
  V v[ROWS_AHEAD];
#pragma unroll
  for (int q = 0; q < ROWS_AHEAD; ++q) {
    const int i = (part * ROWS_AHEAD + q) * 32 + lane;
    if (i < vectors) v[q] = load_vec<V>(x + token * vectors + i);
  }
  for (int j = 0; j < k; ++j) {
    const long long to = __shfl_sync(FULL, row, j);
    if (to < 0) continue;
#pragma unroll
    for (int q = 0; q < ROWS_AHEAD; ++q) {
      const int i = (part * ROWS_AHEAD + q) * 32 + lane;
      if (i < vectors) rows[to * vectors + i] = v[q];
    }
  }
  if (part != 0) return;
  for (int i = lane; i - lane < scales; i += 32) {
    const float f = i < scales ? scale[token * scales + i] : 0.0f;
    for (int j = 0; j < k; ++j) {
      const long long to = __shfl_sync(FULL, row, j);
      if (to >= 0 && i < scales) row_scale[to * scales + i] = f;
    }
  }
}

cudaError_t run_tokens_to_rows(int G, int T, int k, int row_bytes, int scales, const void* x, const float* scale, const int32_t* slot,
                               void* rows, float* row_scale, cudaStream_t stream) {
  const long long tokens = (long long)G * T;
  if (tokens == 0) return cudaSuccess;
  const auto with_vector = [&](auto vec) {
    using V = decltype(vec);
    const int vectors = row_bytes / (int)sizeof(V), parts = (vectors + 32 * ROWS_AHEAD - 1) / (32 * ROWS_AHEAD);
    return launch(scatter_kernel<V>, (tokens * parts + ROWS_WARPS - 1) / ROWS_WARPS, 32 * ROWS_WARPS, 0, stream, tokens, T, k, vectors, parts,
                  scales, static_cast<const V*>(x), scale, slot, static_cast<V*>(rows), row_scale);
  };
  return row_bytes % 16 == 0 ? with_vector(uint4()) : with_vector(uint2());
}

template <typename T>
__global__ void __launch_bounds__(32 * ROWS_WARPS) gather_kernel(long long tokens, int per, int k, int vectors, int parts,
                                                                 const uint4* __restrict__ rows, const int32_t* __restrict__ slot,
                                                                 const float* __restrict__ weights, const uint4* add, uint4* y) {
  constexpr int COUNT = Vec<T>::COUNT;
  const int lane = threadIdx.x & 31;
  const long long item = (long long)blockIdx.x * ROWS_WARPS + (threadIdx.x >> 5), token = item / parts;
  if (token >= tokens) return;
  const int i = (int)(item % parts) * 32 + lane;
  const bool in = i < vectors;
  const long long row = lane < k ? row_of(slot, token * k + lane, token / per, per * k) : -1;
  const float weight = lane >= k ? 0.0f : weights != nullptr ? weights[token * k + lane] : 1.0f;
  float sum[COUNT];
#pragma unroll
  for (int e = 0; e < COUNT; ++e) sum[e] = 0.0f;
  if (add != nullptr && in) Vec<T>::unpack(load_once(add + token * vectors + i), sum);
  for (int j0 = 0; j0 < k; j0 += ROWS_AHEAD) {
    uint4 v[ROWS_AHEAD];
    float w[ROWS_AHEAD];
    long long from[ROWS_AHEAD];
#pragma unroll
    for (int q = 0; q < ROWS_AHEAD; ++q) {
      from[q] = __shfl_sync(FULL, row, (j0 + q) & 31);
      w[q] = __shfl_sync(FULL, weight, (j0 + q) & 31);
      if (j0 + q >= k) from[q] = -1;
      if (from[q] >= 0 && in) v[q] = load_once(rows + from[q] * vectors + i);
    }
#pragma unroll
    for (int q = 0; q < ROWS_AHEAD; ++q) {
      if (from[q] < 0 || !in) continue;
      float f[COUNT];
      Vec<T>::unpack(v[q], f);
#pragma unroll
      for (int e = 0; e < COUNT; ++e) sum[e] = fmaf(w[q], f[e], sum[e]);
    }
  }
  if (in) y[token * vectors + i] = Vec<T>::pack(sum);
}

cudaError_t run_rows_to_tokens(int G, int T, int k, int D, int dtype, const void* rows, const int32_t* slot, const float* weights,
                               const void* add, void* y, cudaStream_t stream) {
  const long long tokens = (long long)G * T;
  if (tokens == 0) return cudaSuccess;
  return with_type(dtype, [&](auto type) {
    using V = decltype(type);
    const int vectors = D / Vec<V>::COUNT, parts = (vectors + 31) / 32;
    return launch(gather_kernel<V>, (tokens * parts + ROWS_WARPS - 1) / ROWS_WARPS, 32 * ROWS_WARPS, 0, stream, tokens, T, k, vectors, parts,
                  static_cast<const uint4*>(rows), slot, weights, static_cast<const uint4*>(add), static_cast<uint4*>(y));
  });
}

// Gradients of the weighted sum: drows[slot] = w dy[t], dw = <dy[t], rows[slot]>. A CTA has a token. drows may be rows itself: a vector is
// read by the thread that writes it, before it does.
template <typename T>
__global__ void __launch_bounds__(32 * ROWS_WARPS) gather_backward_kernel(int per, int k, int vectors, const uint4* __restrict__ dy,
                                                                          const uint4* rows, const int32_t* __restrict__ slot,
                                                                          const float* __restrict__ weights, uint4* drows,
                                                                          float* __restrict__ dweights) {
  constexpr int COUNT = Vec<T>::COUNT;
  __shared__ float part[ROWS_WARPS][MOESCHED_MAX_TOP_K];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long token = blockIdx.x;
  for (int j = 0; j < k; ++j) {
    const long long row = row_of(slot, token * k + j, token / per, per * k);
    const float w = weights[token * k + j];
    float dot = 0.0f;
    if (row >= 0)
      for (int i = threadIdx.x; i < vectors; i += blockDim.x) {
        float g[COUNT], f[COUNT];
        Vec<T>::unpack(dy[token * vectors + i], g);
        Vec<T>::unpack(load_once(rows + row * vectors + i), f);
#pragma unroll
        for (int e = 0; e < COUNT; ++e) {
          dot = fmaf(g[e], f[e], dot);
          g[e] *= w;
        }
        drows[row * vectors + i] = Vec<T>::pack(g);
      }
    dot = warp_sum(dot);
    if (lane == 0) part[warp][j] = dot;
  }
  __syncthreads();
  if (threadIdx.x < k) {
    float sum = 0.0f;
    for (int w = 0; w < (int)blockDim.x / 32; ++w) sum += part[w][threadIdx.x];
    dweights[token * k + threadIdx.x] = sum;
  }
}

cudaError_t run_rows_to_tokens_backward(int G, int T, int k, int D, int dtype, const void* dy, const void* rows, const int32_t* slot,
                                        const float* weights, void* drows, float* dweights, cudaStream_t stream) {
  const long long tokens = (long long)G * T;
  if (tokens == 0) return cudaSuccess;
  return with_type(dtype, [&](auto type) {
    using V = decltype(type);
    const int vectors = D / Vec<V>::COUNT, warps = (vectors + 31) / 32;
    return launch(gather_backward_kernel<V>, tokens, 32 * (warps < ROWS_WARPS ? warps : ROWS_WARPS), 0, stream, T, k, vectors,
                  static_cast<const uint4*>(dy), static_cast<const uint4*>(rows), slot, weights, static_cast<uint4*>(drows), dweights);
  });
}

// 8-bit rows to the type: y = q scale, a scale for every `group` columns. Eight values a lane at a time.
template <typename T>
__global__ void __launch_bounds__(32 * ROWS_WARPS) widen_kernel(long long rows, int eights, int parts, int group, int scales,
                                                                const uint2* __restrict__ q, const float* __restrict__ scale,
                                                                T* __restrict__ y) {
  const int lane = threadIdx.x & 31;
  const long long item = (long long)blockIdx.x * ROWS_WARPS + (threadIdx.x >> 5), row = item / parts;
  if (row >= rows) return;
#pragma unroll
  for (int a = 0; a < ROWS_AHEAD; ++a) {
    const int i = ((int)(item % parts) * ROWS_AHEAD + a) * 32 + lane;
    if (i >= eights) break;
    const uint2 v = load_once8(q + row * eights + i);
    const float s = scale[row * scales + i * 8 / group];
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const unsigned word = e < 4 ? v.x : v.y;
      const __half2_raw both = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(word >> (8 * (e & 2))), __NV_E4M3);
      const float2 wide = __half22float2(*reinterpret_cast<const __half2*>(&both));
      f[e] = wide.x * s;
      f[e + 1] = wide.y * s;
    }
    uint4* to = reinterpret_cast<uint4*>(y + (row * eights + i) * 8);
    if constexpr (sizeof(T) == 2) {
      to[0] = Vec<T>::pack(f);
    } else {
      const float lo[4] = {f[0], f[1], f[2], f[3]}, hi[4] = {f[4], f[5], f[6], f[7]};
      to[0] = Vec<T>::pack(lo);
      to[1] = Vec<T>::pack(hi);
    }
  }
}

cudaError_t run_rows_widen(int R, int D, int group, int dtype, const uint8_t* q, const float* scale, void* y, cudaStream_t stream) {
  if (R == 0) return cudaSuccess;
  return with_type(dtype, [&](auto type) {
    using V = decltype(type);
    const int eights = D / 8, parts = (eights + 32 * ROWS_AHEAD - 1) / (32 * ROWS_AHEAD);
    return launch(widen_kernel<V>, ((long long)R * parts + ROWS_WARPS - 1) / ROWS_WARPS, 32 * ROWS_WARPS, 0, stream, (long long)R, eights,
                  parts, group, (D + group - 1) / group, reinterpret_cast<const uint2*>(q), scale, static_cast<V*>(y));
  });
}

}  // namespace moesched
