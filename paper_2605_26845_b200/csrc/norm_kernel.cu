// Root-mean-square norm of tokens, with the residual's addition before it and an output in 8 bits behind it, and its gradients.
//
//   h = x + r, rounded to the type: the residual stream as it is kept, so that the gradients are those of the values that were normed
//   c = 1 / sqrt(sum h^2 / D + eps),  y = h c w
//   q = y / scale in e4m3, scale = max |y| of a group of columns / 448, from y in 32 bits
// A team of warps has a row in registers, from one read to the outputs: V vectors of 16 bytes a thread. The greatest of a group is
// found among the neighbouring lanes that hold it. Memory bounds all of it: 16384 x 7168 bfloat16 with residual and 8 bits 163 us (1.06 GB, 6.5 TB/s), 8191 x 4096
// with residual 43 us (6.3 TB/s), one row of 7168 2.8 us. What counts is how many warps an SM has whose rows are on their way: 64 registers leave it 28 (bfloat16 with both outputs spills 20 bytes,
// fp16 with a residual 52; with 48 registers 211 us; two vectors a thread 224; rows ahead in shared memory, as the gradients have them, 233), and named barriers would leave it four CTAs.
#include <cuda_fp8.h>

#include "token.cuh"

namespace moesched {

constexpr int NORM_THREADS = 512;                               // of a CTA

// Sum over a team of whole warps, in a fixed order. `part` has a float for every warp of the team, and is not written again before the team has
// met once more. `meet` is the barrier, of the team or of all teams.
template <typename Meet>
__device__ __forceinline__ float team_sum(float v, float* part, int warps, int warp_of_team, Meet meet) {
  v = warp_sum(v);
  if (warps == 1) return v;
  if ((threadIdx.x & 31) == 0) part[warp_of_team] = v;
  __syncwarp();
  meet();
  v = 0.0f;
#pragma unroll 4
  for (int w = 0; w < warps; ++w) v += part[w];
  return v;
}

struct NormArgs {
  int rows, D, team_warps, group_shift, groups;                 // 2^group_shift vectors in each of the groups of a row
  float eps;
  const void *x, *residual, *weight;
  void *sum, *y;
  uint8_t* q;
  float *scale, *rstd;
};

__device__ __forceinline__ float most_or_nan(float a, float b) {
  float v;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(v) : "f"(a), "f"(fabsf(b)));
  return v;
}

// -y / s as 32 bits have it, rounded to nearest, with minus = -1 / s: a product, and what its remainder, which one instruction gives exactly, adds to it (P. Markstein,
// "Computation of elementary functions on the IBM RISC System/6000 processor", 1990). What is rounded to 8 bits then is the nearest to y over the scale; by the product alone
// one value in 37000 was the neighbour. (Negative, so that zeros keep their sign.)
__device__ __forceinline__ Two minus_quotient(Two y, Two s, Two minus) {
  const Two q = mul2(y, minus);
  return fma2(fma2(q, s, y), minus, q);
}

// Vector i of a row: h, of which y and q are made, and where they go. All lanes of a warp come here, those without a vector with zeros.
template <typename T, bool QUANT>
__device__ __forceinline__ void norm_out(const NormArgs& a, const uint4& h, const uint4& w, float c, bool in, size_t row, int i) {
  constexpr int COUNT = Vec<T>::COUNT;
  Two x[COUNT / 2], u[COUNT / 2];
  pairs_of<T>(h, x);
  pairs_of<T>(w, u);
  float f[COUNT];
#pragma unroll
  for (int e = 0; e < COUNT / 2; ++e) {
    x[e] = mul2(mul2(x[e], two(c, c)), u[e]);
    const float2 y = apart_of(x[e]);
    f[2 * e] = y.x;
    f[2 * e + 1] = y.y;
  }
  const size_t at = row * a.D + (size_t)i * COUNT;
  if (a.y != nullptr && in) *reinterpret_cast<uint4*>(static_cast<T*>(a.y) + at) = Vec<T>::pack(f);
  if constexpr (QUANT) {
    float most = fabsf(f[0]);                                   // a NaN stays
#pragma unroll
    for (int e = 1; e < COUNT; ++e) most = most_or_nan(most, f[e]);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1)
      if (o >> a.group_shift == 0) most = most_or_nan(most, __shfl_xor_sync(FULL, most, o));
    // The scale, 2^-126 at least. (A quotient would have one rounding less, which counts for nothing: the values are divided by the scale as it is.) Groups of next to nothing are
    // divided with both sides made larger, so that the remainders are numbers of 32 bits; what is finite is 0 over infinity, and infinity itself NaN.
    float s = most * (1.0f / 448.0f), over = s, by = s;
    if (most < 0x1p-60f) {
      s = fmaxf(s, 0x1p-126f);
      over = by = s * 0x1p80f;
#pragma unroll
      for (int e = 0; e < COUNT / 2; ++e) x[e] = mul2(x[e], two(0x1p80f, 0x1p80f));
    } else if (most == INFINITY) {
      by = 0.0f;
    }
    float minus = -__fdividef(1.0f, over);
    minus = fmaf(fmaf(minus, by, 1.0f), minus, minus);
#pragma unroll
    for (int e = 0; e < COUNT / 2; ++e) {
      const float2 v = apart_of(minus_quotient(x[e], two(by, by), two(minus, minus)));
      f[2 * e] = v.x;
      f[2 * e + 1] = v.y;
    }
    if (in) {
      unsigned packed[COUNT / 4];
#pragma unroll
      for (int e = 0; e < COUNT; e += 4) {
        const unsigned lo = __nv_cvt_float2_to_fp8x2(make_float2(f[e], f[e + 1]), __NV_SATFINITE, __NV_E4M3);
        const unsigned hi = __nv_cvt_float2_to_fp8x2(make_float2(f[e + 2], f[e + 3]), __NV_SATFINITE, __NV_E4M3);
        packed[e / 4] = (lo | hi << 16) ^ 0x80808080u;
      }
      if constexpr (COUNT == 8) *reinterpret_cast<uint2*>(a.q + at) = make_uint2(packed[0], packed[1]);
      else *reinterpret_cast<unsigned*>(a.q + at) = packed[0];
      if ((i & ((1 << a.group_shift) - 1)) == 0) a.scale[row * a.groups + (i >> a.group_shift)] = s;
    }
  }
}

// Vector of h, and what it adds to the sum of squares
template <typename T>
__device__ __forceinline__ uint4 norm_in(const uint4& x, const uint4& r, bool residual, float& total) {
  constexpr int COUNT = Vec<T>::COUNT;
  uint4 h = x;
  float f[COUNT];
  Vec<T>::unpack(x, f);
  if (residual) {
    float g[COUNT];
    Vec<T>::unpack(r, g);
#pragma unroll
    for (int e = 0; e < COUNT; ++e) f[e] += g[e];
    h = Vec<T>::pack(f);
    Vec<T>::unpack(h, f);
  }
#pragma unroll
  for (int e = 0; e < COUNT; ++e) total = fmaf(f[e], f[e], total);
  return h;
}

template <typename T, int V, bool ADDED, bool QUANT>
__global__ void __launch_bounds__(V == 4 ? NORM_THREADS : 256, V == 4 ? 2 : 4) norm_kernel(NormArgs a) {
  __shared__ float part[NORM_THREADS / 32];
  const int vectors = a.D / Vec<T>::COUNT, warps = a.team_warps, threads = 32 * warps;
  const int team = threadIdx.x / threads, at = threadIdx.x - team * threads;
  const long long mine = (long long)blockIdx.x * (blockDim.x / threads) + team;
  const bool active = mine < a.rows;
  const size_t row = active ? (size_t)mine : 0, first = row * vectors;
  const uint4 *x = static_cast<const uint4*>(a.x) + first, *residual = static_cast<const uint4*>(a.residual) + first, zero = make_uint4(0u, 0u, 0u, 0u);
  uint4 h[V], r[V], w[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int i = at + v * threads;
    const bool in = active && i < vectors;
    h[v] = in ? load_once(x + i) : zero;
    r[v] = ADDED && in ? load_once(residual + i) : zero;
  }
  float total = 0.0f;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int i = at + v * threads;
    h[v] = norm_in<T>(h[v], r[v], ADDED, total);
    if (ADDED && active && i < vectors) static_cast<uint4*>(a.sum)[first + i] = h[v];
    w[v] = i < vectors ? __ldg(static_cast<const uint4*>(a.weight) + i) : zero;
  }
  total = team_sum(total, part + team * warps, warps, at >> 5, [] { __syncthreads(); });
  const float c = rsqrtf(total / (float)a.D + a.eps);
  if (a.rstd != nullptr && active && at == 0) a.rstd[row] = c;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int i = at + v * threads;
    norm_out<T, QUANT>(a, h[v], w[v], c, active && i < vectors, row, i);
  }
}

// Few rows, a row a CTA of as many threads as there are vectors: nothing but latency
template <typename T, bool ADDED, bool QUANT>
__global__ void __launch_bounds__(1024) norm_few_kernel(NormArgs a) {
  __shared__ float part[32];
  const int vectors = a.D / Vec<T>::COUNT, i = threadIdx.x;
  const size_t row = blockIdx.x, at = row * vectors + i;
  const bool in = i < vectors;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u), x = in ? load_once(static_cast<const uint4*>(a.x) + at) : zero,
              r = in && ADDED ? load_once(static_cast<const uint4*>(a.residual) + at) : zero,
              w = in ? __ldg(static_cast<const uint4*>(a.weight) + i) : zero;
  float total = 0.0f;
  const uint4 h = norm_in<T>(x, r, ADDED, total);
  if (ADDED && in) static_cast<uint4*>(a.sum)[at] = h;
  total = team_sum(total, part, blockDim.x >> 5, i >> 5, [] { __syncthreads(); });
  const float c = rsqrtf(total / (float)a.D + a.eps);
  if (a.rstd != nullptr && i == 0) a.rstd[row] = c;
  norm_out<T, QUANT>(a, h, w, c, in, row, i);
}

// Rows that are longer than 512 threads hold: one a CTA, read twice, the second time from the L2
template <typename T, bool QUANT>
__global__ void __launch_bounds__(NORM_THREADS) norm_wide_kernel(NormArgs a) {
  constexpr int COUNT = Vec<T>::COUNT;
  __shared__ float part[32];
  const int vectors = a.D / COUNT;
  const size_t row = blockIdx.x;
  const T *x = static_cast<const T*>(a.x) + row * a.D, *residual = static_cast<const T*>(a.residual) + row * a.D;
  T* sum = static_cast<T*>(a.sum) + row * a.D;
  const bool added = a.residual != nullptr;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  float total = 0.0f;
  for (int i = threadIdx.x; i < vectors; i += NORM_THREADS) {
    const uint4 h = norm_in<T>(load_once(x + (size_t)i * COUNT), added ? load_once(residual + (size_t)i * COUNT) : zero, added, total);
    if (added) *reinterpret_cast<uint4*>(sum + (size_t)i * COUNT) = h;
  }
  total = team_sum(total, part, NORM_THREADS / 32, threadIdx.x >> 5, [] { __syncthreads(); });
  const float c = rsqrtf(total / (float)a.D + a.eps);
  if (a.rstd != nullptr && threadIdx.x == 0) a.rstd[row] = c;
  const T* h = added ? sum : x;                                 // (its own stores of before)
  for (int base = 0; base < vectors; base += NORM_THREADS) {
    const int i = base + threadIdx.x;
    const bool in = i < vectors;
    norm_out<T, QUANT>(a, in ? load_once(h + (size_t)i * COUNT) : zero, in ? __ldg(static_cast<const uint4*>(a.weight) + i) : zero, c, in, row, i);
  }
}

template <typename T, int V, bool ADDED, bool QUANT>
static cudaError_t launch_norm_rows(NormArgs a, cudaStream_t stream) {
  const int vectors = a.D / Vec<T>::COUNT;
  a.team_warps = (vectors + 32 * V - 1) / (32 * V);
  const int teams = a.team_warps >= 8 ? 1 : 8 / a.team_warps;
  return launch(norm_kernel<T, V, ADDED, QUANT>, dim3((unsigned)((a.rows + teams - 1) / teams)), dim3(32 * a.team_warps * teams), 0, false, stream, a);
}

// Few rows leave SMs without one, and take the less time the more threads they have: with a vector a thread and with four, 2.9 and 3.5 us for one row of 7168, 3.3 and 3.8 for 148,
// 4.6 both for 222, 7.9 and 6.7 for 592; of 2048 columns (two vectors a thread) 2.0 and 3.3, 2.2 and 3.6, 2.4 and 3.6, 3.2 and 3.7. Short rows
// would leave threads without a vector (300000 x 256 with one vector a thread 95 us, with four 149).
template <typename T, bool ADDED, bool QUANT>
static cudaError_t launch_norm(const NormArgs& a, cudaStream_t stream) {
  const int vectors = a.D / Vec<T>::COUNT;
  if (a.rows <= sm_count() && vectors <= 1024)
    return launch(norm_few_kernel<T, ADDED, QUANT>, dim3(a.rows), dim3((vectors + 31) / 32 * 32), 0, false, stream, a);
  if (vectors <= 32) return launch_norm_rows<T, 1, ADDED, QUANT>(a, stream);
  if (vectors <= 64) return launch_norm_rows<T, 2, ADDED, QUANT>(a, stream);
  if (vectors <= 4 * NORM_THREADS) return launch_norm_rows<T, 4, ADDED, QUANT>(a, stream);
  return launch(norm_wide_kernel<T, QUANT>, dim3(a.rows), dim3(NORM_THREADS), 0, false, stream, a);
}

cudaError_t run_norm(int rows, int D, int dtype, float eps, int group, const void* x, const void* residual, const void* weight,
                     void* sum, void* y, uint8_t* q, float* scale, float* rstd, cudaStream_t stream) {
  NormArgs a{rows, D, 0, 0, q != nullptr ? (D + group - 1) / group : 0, eps, x, residual, weight, sum, y, q, scale, rstd};
  return with_type(dtype, [&](auto type) {
    using T = decltype(type);
    while (q != nullptr && Vec<T>::COUNT << a.group_shift < group) ++a.group_shift;
    if (residual != nullptr) return q != nullptr ? launch_norm<T, true, true>(a, stream) : launch_norm<T, true, false>(a, stream);
    return q != nullptr ? launch_norm<T, false, true>(a, stream) : launch_norm<T, false, false>(a, stream);
  });
}

// Gradients, from g = dy w:  dx = c (g - h c^2 sum(g h) / D) + what comes in for h,  dw = sum over the rows of dy h c.
// A CTA stays on every SM. Its teams take every so many rows, each thread the same 16 columns of all of them, whose dw it has in registers. The vectors of the
// next rows are on their way to the thread's own places in shared memory meanwhile, so that no warp waits for memory between the sums
// of rows. A second kernel adds the dw of the CTAs up, in their order. Rows of more than 8192 columns (SPLIT) have their sums made by a kernel of its own, and a
// CTA has a block of columns.
// Memory bounds it: 8191 x 4096 bfloat16 with dsum 44 us (268 MB, 6.0 TB/s; 3 of it the second kernel), 16384 x 7168 142 us, of 12288 columns 0.67 of that rate. Loaded
// when a row's turn comes 91 us; with two CTAs of 64 registers on an SM, 40 bytes of them spilled, and products one by one 58.
constexpr int NORM_PARTS_VECTORS = 2 * NORM_THREADS / 32 / 4;   // sums of warps, in front of the rows on their way
// Rows on their way, as many as fit: a thread has 16 V bytes for each of three tensors
template <int V>
constexpr int NORM_STAGES = V <= 2 ? 3 : 2;

struct NormBackwardArgs {
  int rows, D, team_warps;
  const void *dy, *h, *weight;
  const float* rstd;
  const void* dsum;
  void* dx;
  float *partial, *dot;
};

template <typename T, int V, bool SPLIT>
__global__ void __launch_bounds__(NORM_THREADS) norm_backward_kernel(NormBackwardArgs a) {
  constexpr int COUNT = Vec<T>::COUNT, PAIRS = COUNT / 2;
  constexpr int STAGES = NORM_STAGES<V>;
  extern __shared__ __align__(16) uint4 shared[];
  float(*part)[NORM_THREADS / 32] = reinterpret_cast<float(*)[NORM_THREADS / 32]>(shared);      // [2]
  uint4* ring = shared + NORM_PARTS_VECTORS;                    // [stage][dy, h, dsum][V][threads of the CTA]
  const int vectors = a.D / COUNT, warps = a.team_warps, threads = 32 * warps, teams = blockDim.x / threads;
  const int team = threadIdx.x / threads, at = threadIdx.x - team * threads, first = SPLIT ? blockIdx.y * V * threads : 0;
  const int tensors = a.dsum != nullptr ? 3 : 2, stage_vectors = tensors * V * blockDim.x, step = gridDim.x * teams;
  const uint4* const from[3] = {static_cast<const uint4*>(a.dy), static_cast<const uint4*>(a.h), static_cast<const uint4*>(a.dsum)};
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  const auto place = [&](int stage, int tensor, int v) { return ring + stage * stage_vectors + (tensor * V + v) * blockDim.x + threadIdx.x; };
  const auto ask = [&](int row, int stage, int t) {
    if (row >= a.rows) return;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int i = first + at + v * threads;
      if (i < vectors) copy_behind(place(stage, t, v), from[t] + (size_t)row * vectors + i);
    }
  };
  Two w[V][PAIRS], dw[V][PAIRS];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int i = first + at + v * threads;
    pairs_of<T>(i < vectors ? __ldg(static_cast<const uint4*>(a.weight) + i) : zero, w[v]);
#pragma unroll
    for (int e = 0; e < PAIRS; ++e) dw[v][e] = two(0.0f, 0.0f);
  }
  int row = blockIdx.x * teams + team;
#pragma unroll
  for (int s = 0; s < STAGES; ++s) {
    for (int t = 0; t < tensors; ++t) ask(row + s * step, s, t);
    copies_asked();
  }
  float next_c = row < a.rows ? a.rstd[row] : 0.0f;
  for (int stage = 0, turn = 0; row < a.rows; row += step, turn ^= 1, stage = stage + 1 == STAGES ? 0 : stage + 1) {
    const float c = next_c;
    if (row + step < a.rows) next_c = a.rstd[row + step];
    copies_here<STAGES - 1>();
    Two gw[V][PAIRS], x[V][PAIRS], sum = two(0.0f, 0.0f);
    const Two cc = two(c, c);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const bool in = first + at + v * threads < vectors;
      Two g[PAIRS];
      pairs_of<T>(in ? *place(stage, 0, v) : zero, g);
      pairs_of<T>(in ? *place(stage, 1, v) : zero, x[v]);
#pragma unroll
      for (int e = 0; e < PAIRS; ++e) {
        gw[v][e] = mul2(g[e], w[v][e]);
        if constexpr (!SPLIT) sum = fma2(gw[v][e], x[v][e], sum);
        dw[v][e] = fma2(mul2(g[e], cc), x[v][e], dw[v][e]);
      }
    }
    ask(row + STAGES * step, stage, 0);
    ask(row + STAGES * step, stage, 1);
    // (two sets of parts in turn: a team that has met for one sum may begin the next while some of it still read)
    float total;
    if constexpr (SPLIT) {
      total = a.dot[row];
    } else {
      const float2 halves = apart_of(sum);
      total = team_sum(halves.x + halves.y, part[turn] + team * warps, warps, at >> 5,
                       [&] { asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(threads) : "memory"); });
    }
    const float along = -total / (float)a.D * c * c;
    const Two against = two(along, along);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int i = first + at + v * threads;
      if (i >= vectors) continue;
      Two s[PAIRS];
      pairs_of<T>(tensors == 3 ? *place(stage, 2, v) : zero, s);
      float f[COUNT];
#pragma unroll
      for (int e = 0; e < PAIRS; ++e) {
        const float2 d = apart_of(fma2(cc, fma2(against, x[v][e], gw[v][e]), s[e]));
        f[2 * e] = d.x;
        f[2 * e + 1] = d.y;
      }
      static_cast<uint4*>(a.dx)[(size_t)row * vectors + i] = Vec<T>::pack(f);
    }
    if (tensors == 3) ask(row + STAGES * step, stage, 2);
    copies_asked();
  }
  copies_here<0>();
  let_next_start();
  // the teams' columns one after the other, in the ring's memory
  float* joined = reinterpret_cast<float*>(ring);
  for (int t = 0; t < teams; ++t) {
    __syncthreads();
    if (team != t) continue;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int i = at + v * threads;
      if (first + i >= vectors) continue;
      float4* mine = reinterpret_cast<float4*>(joined + i * COUNT);
      float4* out = reinterpret_cast<float4*>(a.partial + (size_t)blockIdx.x * a.D + (size_t)(first + i) * COUNT);
#pragma unroll
      for (int e = 0; e < COUNT / 4; ++e) {
        const float2 lo = apart_of(dw[v][2 * e]), hi = apart_of(dw[v][2 * e + 1]);
        float4 value = make_float4(lo.x, lo.y, hi.x, hi.y);
        if (t > 0) {
          const float4 before = mine[e];
          value = make_float4(before.x + value.x, before.y + value.y, before.z + value.z, before.w + value.w);
        }
        if (t + 1 == teams) out[e] = value;
        else mine[e] = value;
      }
    }
  }
}

// sum(g h) of a row a CTA
template <typename T>
__global__ void __launch_bounds__(NORM_THREADS) norm_dot_kernel(int vectors, const uint4* dy, const uint4* h, const uint4* __restrict__ weight,
                                                                float* __restrict__ dot) {
  constexpr int COUNT = Vec<T>::COUNT;
  __shared__ float part[NORM_THREADS / 32];
  const size_t row = blockIdx.x;
  float total = 0.0f;
  for (int i = threadIdx.x; i < vectors; i += NORM_THREADS) {
    float g[COUNT], x[COUNT], w[COUNT];
    Vec<T>::unpack(load_once(dy + row * vectors + i), g);
    Vec<T>::unpack(load_once(h + row * vectors + i), x);
    Vec<T>::unpack(__ldg(weight + i), w);
#pragma unroll
    for (int e = 0; e < COUNT; ++e) total = fmaf(g[e] * w[e], x[e], total);
  }
  total = team_sum(total, part, NORM_THREADS / 32, threadIdx.x >> 5, [] { __syncthreads(); });
  if (threadIdx.x == 0) dot[row] = total;
}

constexpr int COLUMN_ROWS = 16;

// out[d] = sum of partial[.][d] in a fixed order: 32 columns and 16 stretches of the CTAs' sums a CTA
template <typename T>
__global__ void __launch_bounds__(32 * COLUMN_ROWS) column_sum_kernel(int parts, int D, const float* partial, T* out) {
  __shared__ float sums[COLUMN_ROWS][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, d = 32 * blockIdx.x + lane;
  wait_for_previous();
  float total = 0.0f;
  if (d < D) {
#pragma unroll 4
    for (int p = warp; p < parts; p += COLUMN_ROWS) total += partial[(size_t)p * D + d];
  }
  sums[warp][lane] = total;
  __syncthreads();
  if (warp == 0 && d < D) {
    for (int w = 1; w < COLUMN_ROWS; ++w) total += sums[w][lane];
    put(out + d, total);
  }
}

constexpr int NORM_PARTS = 148;                                 // CTAs that sum up dw, at most, whatever the GPU has
static int norm_parts(int rows) { return rows < NORM_PARTS ? rows : NORM_PARTS; }
size_t norm_scratch_bytes(int rows, int D) {
  return ((size_t)norm_parts(rows) * D + (D > 16 * NORM_THREADS ? rows : 0)) * sizeof(float);
}

template <typename T, int V, bool SPLIT>
static cudaError_t launch_norm_backward_rows(NormBackwardArgs a, int& parts, cudaStream_t stream) {
  const int vectors = a.D / Vec<T>::COUNT, tensors = a.dsum != nullptr ? 3 : 2, blocks = SPLIT ? (vectors + V * NORM_THREADS - 1) / (V * NORM_THREADS) : 1;
  a.team_warps = (vectors + 32 * V * blocks - 1) / (32 * V * blocks);
  // as many rows at a time as the CTA's threads take, but not more than leave every SM one
  int teams = NORM_THREADS / 32 / a.team_warps;
  const int most = NORM_PARTS / blocks;
  while (teams > 1 && (long long)(teams - 1) * most >= a.rows) --teams;
  parts = (a.rows + teams - 1) / teams;
  if (parts > most) parts = most;
  const size_t ring = (size_t)NORM_STAGES<V> * tensors * V * 32 * a.team_warps * teams;
  return launch(norm_backward_kernel<T, V, SPLIT>, dim3(parts, blocks), dim3(32 * a.team_warps * teams), 16 * (NORM_PARTS_VECTORS + ring), false,
                stream, a);
}

// 16 values of a row a thread, half of them where the row has no more than 256 (300000 x 256: 104 us, 219 before rows were ahead)
template <typename T>
static cudaError_t launch_norm_backward(const NormBackwardArgs& a, int& parts, cudaStream_t stream) {
  constexpr int V = 16 / Vec<T>::COUNT;
  const int vectors = a.D / Vec<T>::COUNT;
  if (vectors <= 16 * V) return launch_norm_backward_rows<T, V / 2, false>(a, parts, stream);
  if (vectors <= V * NORM_THREADS) return launch_norm_backward_rows<T, V, false>(a, parts, stream);
  const cudaError_t e = launch(norm_dot_kernel<T>, dim3(a.rows), dim3(NORM_THREADS), 0, false, stream, vectors, static_cast<const uint4*>(a.dy),
                               static_cast<const uint4*>(a.h), static_cast<const uint4*>(a.weight), a.dot);
  return e != cudaSuccess ? e : launch_norm_backward_rows<T, V, true>(a, parts, stream);
}

cudaError_t run_norm_backward(int rows, int D, int dtype, const void* dy, const void* h, const void* weight, const float* rstd,
                              const void* dsum, void* dx, void* dweight, float* scratch, cudaStream_t stream) {
  return with_type(dtype, [&](auto type) {
    using T = decltype(type);
    int parts = 0;
    if (rows > 0) {
      const NormBackwardArgs a{rows, D, 0, dy, h, weight, rstd, dsum, dx, scratch, scratch + (size_t)norm_parts(rows) * D};
      if (cudaError_t e = launch_norm_backward<T>(a, parts, stream); e != cudaSuccess) return e;
    }
    return launch(column_sum_kernel<T>, dim3((unsigned)((D + 31) / 32)), dim3(32 * COLUMN_ROWS), 0, true, stream, parts, D,
                  static_cast<const float*>(scratch), static_cast<T*>(dweight));
  });
}

}  // namespace moesched
