// Tokens to the rows of the send buffer and back: rows[slot[t k + j]] = x[t], and y[t] = sum_j w_tj rows[slot[t k + j]].
//
// A choice whose slot is not one of the source's T k rows was not sent: it writes nothing and adds nothing. Everything is done token by token, so
// that a token's row is read once for all of its choices, sums are in the order of the choices, and nothing needs the inverse of `slot`.
// A warp has a part of a token's row; memory bounds all of it, so what counts is that enough is on its way.
#include <cuda_fp8.h>

#include "token.cuh"

namespace moesched {

constexpr int ROWS_WARPS = 4;      // of a CTA

// A CTA is a box of warps: y the parts of a row that it has, z tokens side by side. Rows of more parts take several CTAs, next to one another.
struct RowsGrid {
  int blocks;                      // CTAs of a token
  dim3 ctas, threads;
};
static RowsGrid rows_grid(long long tokens, int parts, int warps = ROWS_WARPS) {
  RowsGrid g;
  g.blocks = (parts + warps - 1) / warps;
  const int y = (parts + g.blocks - 1) / g.blocks, z = warps / y;
  g.threads = dim3(32, y, z);
  g.ctas = dim3((unsigned)((tokens + z - 1) / z * g.blocks));
  return g;
}
struct RowsPlace {
  unsigned token;
  int part;
};
__device__ __forceinline__ RowsPlace rows_place(int blocks) {
  const unsigned set = blocks == 1 ? blockIdx.x : blockIdx.x / (unsigned)blocks;
  return {set * blockDim.z + threadIdx.z, (int)((blockIdx.x - set * blocks) * blockDim.y + threadIdx.y)};
}

// Rows of the token's choices, one a lane, counted from the first source; negative: not sent
__device__ __forceinline__ long long row_of(const int32_t* slot, unsigned token, int k, int per, int j, bool wanted) {
  if (!wanted) return -1;
  const int at = slot[(long long)token * k + j], rows = per * k;
  return (unsigned)at < (unsigned)rows ? (long long)(token / (unsigned)per) * rows + at : -1;
}

template <typename V>
__device__ __forceinline__ V load_vec(const void* p) {
  if constexpr (sizeof(V) == 16) return load_once(p);
  else return load_once8(p);
}

template <typename V, int AHEAD>
__global__ void __launch_bounds__(32 * ROWS_WARPS) scatter_kernel(unsigned tokens, int per, int k, int vectors, int blocks, int scales,
                                                                  const V* __restrict__ x, const float* __restrict__ scale,
                                                                  const int32_t* __restrict__ slot, V* __restrict__ rows,
                                                                  float* __restrict__ row_scale) {
  const int lane = threadIdx.x;
  const auto [token, part] = rows_place(blocks);
  if (token >= tokens) return;
  V v[AHEAD];
#pragma unroll
  for (int q = 0; q < AHEAD; ++q) {
    const int i = (part * AHEAD + q) * 32 + lane;
    if (i < vectors) v[q] = load_vec<V>(x + (size_t)token * vectors + i);
  }
  const long long row = row_of(slot, token, k, per, lane, lane < k);
#pragma unroll 4
  for (int j = 0; j < k; ++j) {
    const long long to = __shfl_sync(FULL, row, j);
    if (to < 0) continue;
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) {
      const int i = (part * AHEAD + q) * 32 + lane;
      if (i < vectors) rows[to * vectors + i] = v[q];
    }
  }
  if (part != 0) return;
  for (int i = lane; i - lane < scales; i += 32) {
    const float f = i < scales ? scale[(size_t)token * scales + i] : 0.0f;
    for (int j = 0; j < k; ++j) {
      const long long to = __shfl_sync(FULL, row, j);
      if (to >= 0 && i < scales) row_scale[to * scales + i] = f;
    }
  }
}

// whether there are so few warps that they should rather have less each
static bool few_warps(long long warps) { return warps < 8LL * sm_count(); }

cudaError_t run_tokens_to_rows(int G, int T, int k, int row_bytes, int scales, const void* x, const float* scale, const int32_t* slot,
                               void* rows, float* row_scale, cudaStream_t stream) {
  const unsigned tokens = (unsigned)G * T;
  const auto with = [&](auto vec, auto ahead) {
    using V = decltype(vec);
    constexpr int AHEAD = decltype(ahead)::value;
    const int vectors = row_bytes / (int)sizeof(V), parts = (vectors + 32 * AHEAD - 1) / (32 * AHEAD);
    const RowsGrid g = rows_grid(tokens, parts);
    return launch(scatter_kernel<V, AHEAD>, g.ctas, g.threads, 0, false, stream, tokens, T, k, vectors, g.blocks, scales,
                  static_cast<const V*>(x), scale, slot, static_cast<V*>(rows), row_scale);
  };
  const bool few = few_warps((long long)tokens * ((row_bytes + 2047) / 2048));
  if (row_bytes % 16 == 0)
    return few ? with(uint4(), std::integral_constant<int, 1>()) : with(uint4(), std::integral_constant<int, 4>());
  return few ? with(uint2(), std::integral_constant<int, 1>()) : with(uint2(), std::integral_constant<int, 4>());
}

// ROWS rows at a time, VECTORS vectors of each a lane
template <typename T, int ROWS, int VECTORS>
__global__ void __launch_bounds__(32 * ROWS_WARPS) gather_kernel(unsigned tokens, int per, int k, int vectors, int blocks,
                                                                 const uint4* __restrict__ rows, const int32_t* __restrict__ slot,
                                                                 const float* __restrict__ weights, const uint4* add, uint4* y) {
  constexpr int COUNT = Vec<T>::COUNT;
  const int lane = threadIdx.x;
  const auto [token, part] = rows_place(blocks);
  if (token >= tokens) return;
  const int i0 = part * VECTORS * 32 + lane;
  const long long row = row_of(slot, token, k, per, lane, lane < k);
  const float weight = lane >= k ? 0.0f : weights != nullptr ? weights[(size_t)token * k + lane] : 1.0f;
  float sum[VECTORS][COUNT];
#pragma unroll
  for (int a = 0; a < VECTORS; ++a) {
#pragma unroll
    for (int e = 0; e < COUNT; ++e) sum[a][e] = 0.0f;
    if (add != nullptr && i0 + 32 * a < vectors) Vec<T>::unpack(load_once(add + (size_t)token * vectors + i0 + 32 * a), sum[a]);
  }
  for (int j0 = 0; j0 < k; j0 += ROWS) {
    uint4 v[ROWS][VECTORS];
    long long from[ROWS];
#pragma unroll
    for (int q = 0; q < ROWS; ++q) {
      from[q] = __shfl_sync(FULL, row, (j0 + q) & 31);
      if (j0 + q >= k) from[q] = -1;
#pragma unroll
      for (int a = 0; a < VECTORS; ++a)
        if (from[q] >= 0 && i0 + 32 * a < vectors) v[q][a] = load_once(rows + from[q] * vectors + i0 + 32 * a);
    }
#pragma unroll
    for (int q = 0; q < ROWS; ++q) {
      const float w = __shfl_sync(FULL, weight, (j0 + q) & 31);
      if (from[q] < 0) continue;
#pragma unroll
      for (int a = 0; a < VECTORS; ++a) {
        if (i0 + 32 * a >= vectors) continue;
        float f[COUNT];
        Vec<T>::unpack(v[q][a], f);
#pragma unroll
        for (int e = 0; e < COUNT; ++e) sum[a][e] = fmaf(w, f[e], sum[a][e]);
      }
    }
  }
#pragma unroll
  for (int a = 0; a < VECTORS; ++a)
    if (i0 + 32 * a < vectors) y[(size_t)token * vectors + i0 + 32 * a] = Vec<T>::pack(sum[a]);
}

cudaError_t run_rows_to_tokens(int G, int T, int k, int D, int dtype, const void* rows, const int32_t* slot, const float* weights,
                               const void* add, void* y, cudaStream_t stream) {
  const unsigned tokens = (unsigned)G * T;
  return with_type(dtype, [&](auto type) {
    using V = decltype(type);
    const int vectors = D / Vec<V>::COUNT;
    const auto with = [&](auto kern, int count) {
      const RowsGrid g = rows_grid(tokens, (vectors + 32 * count - 1) / (32 * count));
      return launch(kern, g.ctas, g.threads, 0, false, stream, tokens, T, k, vectors, g.blocks, static_cast<const uint4*>(rows), slot,
                    weights, static_cast<const uint4*>(add), static_cast<uint4*>(y));
    };
    if (few_warps((long long)tokens * ((vectors + 31) / 32))) return with(gather_kernel<V, 8, 1>, 1);
    if (k > 4 || vectors <= 32) return with(gather_kernel<V, 4, 1>, 1);
    return with(gather_kernel<V, 4, 2>, 2);
  });
}

// Eight sums over the lanes at once: lane l gets the sum of s[l / 4]. Every step halves what a lane still has.
__device__ __forceinline__ float eight_sums(float (&s)[8]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int half = 4, o = 16; half > 0; half >>= 1, o >>= 1) {
    const bool upper = (lane & o) != 0;
#pragma unroll
    for (int q = 0; q < half; ++q) {
      const float give = upper ? s[q] : s[q + half], keep = upper ? s[q + half] : s[q];
      s[q] = keep + __shfl_xor_sync(FULL, give, o);
    }
  }
  float v = s[0];
  v += __shfl_xor_sync(FULL, v, 2);
  return v + __shfl_xor_sync(FULL, v, 1);
}

// Gradients of the weighted sum: drows[slot] = w dy[t], dw = <dy[t], rows[slot]>. The warps of a token (z: tokens side by side) go over its vectors,
// ROWS rows at a time. drows may be rows itself: a vector is read by the thread that writes it, before it does.
template <typename T, int ROWS>
__global__ void __launch_bounds__(512, ROWS == 8 ? 1 : 2) gather_backward_kernel(unsigned tokens, int per, int k, int vectors, const uint4* dy, const uint4* rows,
                                                              const int32_t* __restrict__ slot, const float* __restrict__ weights,
                                                              uint4* drows, float* __restrict__ dweights) {
  constexpr int COUNT = Vec<T>::COUNT;
  __shared__ float part[16][MOESCHED_MAX_TOP_K];
  const int lane = threadIdx.x, warp = threadIdx.y, warps = blockDim.y;
  const unsigned mine = blockIdx.x * blockDim.z + threadIdx.z, token = mine < tokens ? mine : 0u;
  const bool active = mine < tokens;
  float(*own)[MOESCHED_MAX_TOP_K] = part + threadIdx.z * warps;
  const long long row = row_of(slot, token, k, per, lane, active && lane < k);
  const float weight = active && lane < k ? weights[(size_t)token * k + lane] : 0.0f;
  for (int j0 = 0; j0 < k; j0 += ROWS) {
    long long at[ROWS];
    float sum[8];
#pragma unroll
    for (int q = 0; q < ROWS; ++q) {
      at[q] = __shfl_sync(FULL, row, (j0 + q) & 31);
      if (j0 + q >= k) at[q] = -1;
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) sum[q] = 0.0f;
    for (int i = 32 * warp + lane; i - lane < vectors; i += 32 * warps) {
      const bool in = i < vectors;
      uint4 v[ROWS];
#pragma unroll
      for (int q = 0; q < ROWS; ++q)
        if (at[q] >= 0 && in) v[q] = load_once(rows + at[q] * vectors + i);
      float g[COUNT];
      Vec<T>::unpack(active && in ? dy[(size_t)token * vectors + i] : make_uint4(0u, 0u, 0u, 0u), g);
#pragma unroll
      for (int q = 0; q < ROWS; ++q) {
        const float w = __shfl_sync(FULL, weight, (j0 + q) & 31);
        if (at[q] < 0 || !in) continue;
        float f[COUNT];
        Vec<T>::unpack(v[q], f);
#pragma unroll
        for (int e = 0; e < COUNT; ++e) {
          sum[q] = fmaf(g[e], f[e], sum[q]);
          f[e] = g[e] * w;
        }
        drows[at[q] * vectors + i] = Vec<T>::pack(f);
      }
    }
    const float total = eight_sums(sum);
    if ((lane & 3) == 0 && lane / 4 < ROWS) own[warp][j0 + lane / 4] = total;
  }
  if (warps > 1) __syncthreads();
  else __syncwarp();
  if (warp == 0 && active && lane < k) {
    float total = own[0][lane];
    for (int w = 1; w < warps; ++w) total += own[w][lane];
    dweights[(size_t)token * k + lane] = total;
  }
}

cudaError_t run_rows_to_tokens_backward(int G, int T, int k, int D, int dtype, const void* dy, const void* rows, const int32_t* slot,
                                        const float* weights, void* drows, float* dweights, cudaStream_t stream) {
  const unsigned tokens = (unsigned)G * T;
  return with_type(dtype, [&](auto type) {
    using V = decltype(type);
    const int vectors = D / Vec<V>::COUNT, all = (vectors + 31) / 32;
    const auto with = [&](auto kern, int most) {
      const int turns = (all + most - 1) / most, warps = (all + turns - 1) / turns, z = warps >= 8 ? 1 : 8 / warps;
      return launch(kern, dim3((tokens + z - 1) / z), dim3(32, warps, z), 0, false, stream, tokens, T, k, vectors,
                    static_cast<const uint4*>(dy), static_cast<const uint4*>(rows), slot, weights, static_cast<uint4*>(drows), dweights);
    };
    return few_warps((long long)tokens * all) ? with(gather_backward_kernel<V, 8>, 16) : with(gather_backward_kernel<V, 4>, 8);
  });
}

// 8-bit rows to the type: y = q scale, a scale for every `group` columns. A lane has as many values as 16 bytes of the type hold at a time.
template <typename T, int AHEAD>
__global__ void __launch_bounds__(32 * ROWS_WARPS) widen_kernel(unsigned rows, int vectors, int blocks, int shift, int scales,
                                                                const uint8_t* __restrict__ q, const float* __restrict__ scale,
                                                                uint4* __restrict__ y) {
  constexpr int COUNT = Vec<T>::COUNT, WORDS = COUNT / 4;
  const int lane = threadIdx.x;
  const auto [row, part] = rows_place(blocks);
  if (row >= rows) return;
  unsigned v[AHEAD][WORDS];
  float s[AHEAD];
#pragma unroll
  for (int a = 0; a < AHEAD; ++a) {
    const int i = (part * AHEAD + a) * 32 + lane;
    if (i < vectors) {
      const uint8_t* from = q + ((size_t)row * vectors + i) * COUNT;
      if constexpr (WORDS == 2) {
        const uint2 w = load_once8(from);
        v[a][0] = w.x;
        v[a][1] = w.y;
      } else {
        v[a][0] = load_once4(from);
      }
      s[a] = __ldg(scale + (size_t)row * scales + (i >> shift));
    }
  }
#pragma unroll
  for (int a = 0; a < AHEAD; ++a) {
    const int i = (part * AHEAD + a) * 32 + lane;
    if (i >= vectors) continue;
    float f[COUNT];
#pragma unroll
    for (int e = 0; e < COUNT; e += 2) {
      const __half2_raw both = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(v[a][e / 4] >> (8 * (e & 2))), __NV_E4M3);
      const float2 wide = __half22float2(*reinterpret_cast<const __half2*>(&both));
      f[e] = wide.x * s[a];
      f[e + 1] = wide.y * s[a];
    }
    y[(size_t)row * vectors + i] = Vec<T>::pack(f);
  }
}

cudaError_t run_rows_widen(int R, int D, int group, int dtype, const uint8_t* q, const float* scale, void* y, cudaStream_t stream) {
  return with_type(dtype, [&](auto type) {
    using V = decltype(type);
    constexpr int AHEAD = 4;
    int shift = 0;
    while (Vec<V>::COUNT << shift < group) ++shift;             // vectors of a group: 2^shift
    const int vectors = D / Vec<V>::COUNT;
    const RowsGrid g = rows_grid(R, (vectors + 32 * AHEAD - 1) / (32 * AHEAD));
    return launch(widen_kernel<V, AHEAD>, g.ctas, g.threads, 0, false, stream, (unsigned)R, vectors, g.blocks, shift, (D + group - 1) / group, q,
                  scale, static_cast<uint4*>(y));
  });
}

}  // namespace moesched
