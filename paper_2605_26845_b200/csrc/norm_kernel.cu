// Root-mean-square norm of tokens, with the residual's addition before it and an output in 8 bits behind it, and its gradients.
//
//   h = x + r, rounded to the type: the residual stream as it is kept, so that the gradients are those of the values that were normed
//   c = 1 / sqrt(sum h^2 / D + eps),  y = h c w
//   q = y / scale in e4m3, scale = max |y| of a group of columns / 448, from y in 32 bits
// A team of threads has a row in registers, from one read to the outputs: TEAM threads with V vectors of 16 bytes each. The
// greatest of a group is found among the neighbouring lanes that hold it.
#include <cuda_fp8.h>

#include "token.cuh"

namespace moesched {

constexpr int NORM_THREADS = 1024;

// Sum over a team of whole warps, in a fixed order; `part` has a float for every warp of the CTA. Teams of one warp need no barrier.
__device__ __forceinline__ float team_sum(float v, float* part, int team, int warps) {
  v = warp_sum(v);
  if (warps == 1) return v;
  const int warp = threadIdx.x >> 5;
  if ((threadIdx.x & 31) == 0) part[warp] = v;
  __syncthreads();
  v = 0.0f;
  for (int w = 0; w < warps; ++w) v += part[team * warps + w];
  return v;
}

template <typename T, int V, bool QUANT>
__global__ void __launch_bounds__(NORM_THREADS) norm_kernel(int rows, int D, int team_warps, int group, float eps, const T* x,
                                                            const T* residual, const T* __restrict__ weight, T* sum, T* y,
                                                            uint8_t* q, float* scale, float* rstd) {
  constexpr int COUNT = Vec<T>::COUNT;
  __shared__ float part[NORM_THREADS / 32];
  const int vectors = D / COUNT, threads = 32 * team_warps;
  const int team = threadIdx.x / threads, at = threadIdx.x % threads;
  const long long row = (long long)blockIdx.x * (blockDim.x / threads) + team;
  const bool active = row < rows;
  const size_t first = (size_t)(active ? row : 0) * D;
  uint4 h[V], w[V];
  float total = 0.0f;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int i = at + v * threads;
    const bool in = active && i < vectors;
    h[v] = in ? load_once(x + first + (size_t)i * COUNT) : make_uint4(0u, 0u, 0u, 0u);
    if (residual != nullptr) w[v] = in ? load_once(residual + first + (size_t)i * COUNT) : make_uint4(0u, 0u, 0u, 0u);
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int i = at + v * threads;
    float f[COUNT];
    Vec<T>::unpack(h[v], f);
    if (residual != nullptr) {
      float r[COUNT];
      Vec<T>::unpack(w[v], r);
#pragma unroll
      for (int e = 0; e < COUNT; ++e) f[e] += r[e];
      h[v] = Vec<T>::pack(f);
      Vec<T>::unpack(h[v], f);
      if (active && i < vectors) *reinterpret_cast<uint4*>(sum + first + (size_t)i * COUNT) = h[v];
    }
#pragma unroll
    for (int e = 0; e < COUNT; ++e) total = fmaf(f[e], f[e], total);
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int i = at + v * threads;
    w[v] = i < vectors ? __ldg(reinterpret_cast<const uint4*>(weight) + i) : make_uint4(0u, 0u, 0u, 0u);
  }
  total = team_sum(total, part, team, team_warps);
  const float c = rsqrtf(total / (float)D + eps);
  if (rstd != nullptr && active && at == 0) rstd[row] = c;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int i = at + v * threads;
    const bool in = active && i < vectors;
    float f[COUNT], g[COUNT];
    Vec<T>::unpack(h[v], f);
    Vec<T>::unpack(w[v], g);
#pragma unroll
    for (int e = 0; e < COUNT; ++e) f[e] = f[e] * c * g[e];
    if (y != nullptr && in) *reinterpret_cast<uint4*>(y + first + (size_t)i * COUNT) = Vec<T>::pack(f);
    if constexpr (QUANT) {
      unsigned most = 0u;                                       // (of the magnitudes' bits: a NaN is above infinity, and stays)
#pragma unroll
      for (int e = 0; e < COUNT; ++e) most = max(most, __float_as_uint(f[e]) & 0x7fffffffu);
      for (int o = group / COUNT / 2; o > 0; o >>= 1) most = max(most, __shfl_xor_sync(FULL, most, o));
      // not below the smallest normal number, whose reciprocal is finite: groups of zeros, or of hardly more
      const float top = __uint_as_float(most), s = top < 448.0f * 0x1p-126f ? 0x1p-126f : top / 448.0f, inverse = 1.0f / s;
      if (in) {
        unsigned packed[COUNT / 4];
#pragma unroll
        for (int e = 0; e < COUNT; e += 4) {
          const unsigned lo = __nv_cvt_float2_to_fp8x2(make_float2(f[e] * inverse, f[e + 1] * inverse), __NV_SATFINITE, __NV_E4M3);
          const unsigned hi = __nv_cvt_float2_to_fp8x2(make_float2(f[e + 2] * inverse, f[e + 3] * inverse), __NV_SATFINITE, __NV_E4M3);
          packed[e / 4] = lo | hi << 16;
        }
        uint8_t* to = q + first + (size_t)i * COUNT;
        if constexpr (COUNT == 8) *reinterpret_cast<uint2*>(to) = make_uint2(packed[0], packed[1]);
        else *reinterpret_cast<unsigned*>(to) = packed[0];
        const int per = group / COUNT;
        if (i % per == 0) scale[(size_t)row * ((D + group - 1) / group) + i / per] = s;
      }
    }
  }
}

template <typename T, int V>
static cudaError_t launch_norm(int rows, int D, int group, float eps, const void* x, const void* residual, const void* weight,
                               void* sum, void* y, uint8_t* q, float* scale, float* rstd, cudaStream_t stream) {
  const int vectors = D / Vec<T>::COUNT, warps = (vectors + 32 * V - 1) / (32 * V), teams = warps >= 8 ? 1 : 8 / warps;
  const auto kern = q != nullptr ? norm_kernel<T, V, true> : norm_kernel<T, V, false>;
  return launch(kern, (rows + teams - 1) / teams, 32 * warps * teams, 0, stream, rows, D, warps, group, eps, static_cast<const T*>(x),
                static_cast<const T*>(residual), static_cast<const T*>(weight), static_cast<T*>(sum), static_cast<T*>(y), q, scale, rstd);
}

cudaError_t run_norm(int rows, int D, int dtype, float eps, int group, const void* x, const void* residual, const void* weight,
                     void* sum, void* y, uint8_t* q, float* scale, float* rstd, cudaStream_t stream) {
  if (rows == 0) return cudaSuccess;
  return with_type(dtype, [&](auto type) {
    using T = decltype(type);
    const int vectors = D / Vec<T>::COUNT;
    if (vectors <= 4 * NORM_THREADS) return launch_norm<T, 4>(rows, D, group, eps, x, residual, weight, sum, y, q, scale, rstd, stream);
    return launch_norm<T, 16>(rows, D, group, eps, x, residual, weight, sum, y, q, scale, rstd, stream);
  });
}

// Gradients, from g = dy w:  dx = c (g - h c^2 sum(g h) / D) + what comes in for h,  dw = sum over the rows of dy h c.
// A CTA takes every gridDim-th set of rows and keeps its threads' columns of dw in registers; a second kernel adds the CTAs' up, in
// their order.
template <typename T, int V>
__global__ void __launch_bounds__(NORM_THREADS) norm_backward_kernel(int rows, int D, int team_warps, const T* dy, const T* h,
                                                                     const T* __restrict__ weight, const float* __restrict__ rstd,
                                                                     const T* dsum, T* dx, float* __restrict__ partial) {
  constexpr int COUNT = Vec<T>::COUNT;
  extern __shared__ __align__(16) float joined[];               // [D], where teams share the CTA
  __shared__ float part[2][NORM_THREADS / 32];
  const int vectors = D / COUNT, threads = 32 * team_warps, teams = blockDim.x / threads;
  const int team = threadIdx.x / threads, at = threadIdx.x % threads;
  float dw[V][COUNT];
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < COUNT; ++e) dw[v][e] = 0.0f;
  int set = 0;
  for (long long base = (long long)blockIdx.x * teams; base < rows; base += (long long)gridDim.x * teams, set ^= 1) {
    const long long row = base + team;
    const bool active = row < rows;
    const size_t first = (size_t)(active ? row : 0) * D;
    const float c = active ? rstd[row] : 0.0f;
    uint4 a[V], b[V];
    float total = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int i = at + v * threads;
      const bool in = active && i < vectors;
      a[v] = in ? load_once(dy + first + (size_t)i * COUNT) : make_uint4(0u, 0u, 0u, 0u);
      b[v] = in ? load_once(h + first + (size_t)i * COUNT) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int i = at + v * threads;
      float g[COUNT], x[COUNT], w[COUNT];
      Vec<T>::unpack(a[v], g);
      Vec<T>::unpack(b[v], x);
      Vec<T>::unpack(i < vectors ? __ldg(reinterpret_cast<const uint4*>(weight) + i) : make_uint4(0u, 0u, 0u, 0u), w);
#pragma unroll
      for (int e = 0; e < COUNT; ++e) {
        total = fmaf(g[e] * w[e], x[e], total);
        dw[v][e] = fmaf(g[e] * c, x[e], dw[v][e]);
      }
    }
    total = team_sum(total, part[set], team, team_warps);        // (two sets: the next sum may begin while this one is read)
    const float along = total / (float)D * c * c;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int i = at + v * threads;
      if (!active || i >= vectors) continue;
      float g[COUNT], x[COUNT], w[COUNT], s[COUNT];
      Vec<T>::unpack(a[v], g);
      Vec<T>::unpack(b[v], x);
      Vec<T>::unpack(__ldg(reinterpret_cast<const uint4*>(weight) + i), w);
      if (dsum != nullptr) Vec<T>::unpack(load_once(dsum + first + (size_t)i * COUNT), s);
#pragma unroll
      for (int e = 0; e < COUNT; ++e) {
        g[e] = c * fmaf(-along, x[e], g[e] * w[e]);
        if (dsum != nullptr) g[e] += s[e];
      }
      *reinterpret_cast<uint4*>(dx + first + (size_t)i * COUNT) = Vec<T>::pack(g);
    }
  }
  // the teams' columns one after the other
  for (int t = 0; t < teams; ++t) {
    if (team == t) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int i = at + v * threads;
        if (i >= vectors) continue;
#pragma unroll
        for (int e = 0; e < COUNT; ++e) {
          float* mine = joined + i * COUNT + e;
          const float value = t == 0 ? dw[v][e] : *mine + dw[v][e];
          if (t + 1 == teams) partial[(size_t)blockIdx.x * D + i * COUNT + e] = value;
          else *mine = value;
        }
      }
    }
    if (teams > 1) __syncthreads();
  }
}

constexpr int COLUMN_ROWS = 16;

// out[d] = sum of partial[.][d] in a fixed order: 32 columns and 16 stretches of the CTAs' sums a CTA
template <typename T>
__global__ void __launch_bounds__(32 * COLUMN_ROWS) column_sum_kernel(int parts, int D, const float* __restrict__ partial, T* out) {
  __shared__ float sums[COLUMN_ROWS][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, d = 32 * blockIdx.x + lane;
  float total = 0.0f;
  if (d < D)
    for (int p = warp; p < parts; p += COLUMN_ROWS) total += partial[(size_t)p * D + d];
  sums[warp][lane] = total;
  __syncthreads();
  if (warp == 0 && d < D) {
    for (int w = 1; w < COLUMN_ROWS; ++w) total += sums[w][lane];
    put(out + d, total);
  }
}

static int norm_parts(int rows) { return rows < 2 * 148 ? rows : 2 * 148; }   // CTAs that sum up dw, whatever the GPU has
size_t norm_scratch_bytes(int rows, int D) { return (size_t)norm_parts(rows) * D * sizeof(float); }

template <typename T, int V>
static cudaError_t launch_norm_backward(int rows, int D, const void* dy, const void* h, const void* weight, const float* rstd,
                                        const void* dsum, void* dx, float* partial, cudaStream_t stream) {
  const int vectors = D / Vec<T>::COUNT, warps = (vectors + 32 * V - 1) / (32 * V), teams = warps >= 8 ? 1 : 8 / warps;
  const auto kern = norm_backward_kernel<T, V>;
  const size_t smem = teams > 1 ? (size_t)D * sizeof(float) : 0;
  return launch(kern, norm_parts(rows), 32 * warps * teams, smem, stream, rows, D, warps, static_cast<const T*>(dy),
                static_cast<const T*>(h), static_cast<const T*>(weight), rstd, static_cast<const T*>(dsum), static_cast<T*>(dx), partial);
}

cudaError_t run_norm_backward(int rows, int D, int dtype, const void* dy, const void* h, const void* weight, const float* rstd,
                              const void* dsum, void* dx, void* dweight, float* scratch, cudaStream_t stream) {
  return with_type(dtype, [&](auto type) {
    using T = decltype(type);
    if (rows > 0) {
      const int vectors = D / Vec<T>::COUNT;
      const cudaError_t e =
          vectors <= 2 * NORM_THREADS ? launch_norm_backward<T, 2>(rows, D, dy, h, weight, rstd, dsum, dx, scratch, stream)
                                      : launch_norm_backward<T, 16>(rows, D, dy, h, weight, rstd, dsum, dx, scratch, stream);
      if (e != cudaSuccess) return e;
    }
    return launch(column_sum_kernel<T>, (D + 31) / 32, 32 * COLUMN_ROWS, 0, stream, norm_parts(rows), D, static_cast<const float*>(scratch),
                  static_cast<T*>(dweight));
  });
}

}  // namespace moesched
