// Tokens to the rows of the send buffer and back: rows[slot[t k + j]] = x[t], and y[t] = sum_j w_tj rows[slot[t k + j]].
//
// A choice whose slot is not one of the source's T k rows was not sent: it writes nothing and adds nothing. Everything is done token by token, so
// that a token's row is read once for all of its choices, sums are in the order of the choices, and nothing needs the inverse of `slot`.
// Memory bounds all of it, so what counts is that enough is on its way. Where rows are read, a thread has a vector of 16 bytes of some token, or a few of them,
// and looks the token's slots up itself: no lane is idle at the end of a row, whatever its width. Where rows are written, a warp has a part of one, so that what it
// writes lies together (the other way costs 3 to 10 % there), unless rows are shorter than a warp.
// bfloat16, 8191 tokens of 4096 features, 8 choices: rows 96 us (604 MB, 6.3 TB/s), back 106, gradients 183 (1.14 GB, 6.2 TB/s); 131072 rows of 7168 widened 414 us. 16 tokens of
// 7168: 2.3, 2.9, 5.6 us.
#include <cuda_fp8.h>

#include "token.cuh"

namespace moesched {

constexpr int FLAT_THREADS = 128;

// Vectors of a CTA's threads among those of all tokens, `vectors` each
struct FlatPlace {
  long long at;      // of all
  unsigned token;
  int i;             // of the token's
};
__device__ __forceinline__ FlatPlace flat_place(long long block, int vectors, const FastDiv& by_vectors) {
  const long long at = block * FLAT_THREADS + threadIdx.x, token = fast_div(at, by_vectors);
  return {at, (unsigned)token, (int)(at - token * vectors)};
}
static long long flat_ctas(long long vectors, int each) { return (vectors + FLAT_THREADS * each - 1) / (FLAT_THREADS * each); }

// The sources' rows: `per` tokens with k choices each
struct Sources {
  unsigned tokens;
  int per, k;
  __device__ __forceinline__ unsigned rows() const { return (unsigned)per * k; }
  __device__ __forceinline__ long long first(unsigned token) const {
    return tokens == (unsigned)per ? 0 : (long long)(token / (unsigned)per) * rows();
  }
};

template <typename V>
__device__ __forceinline__ V load_vec(const void* p) {
  if constexpr (sizeof(V) == 16) return load_once(p);
  else if constexpr (sizeof(V) == 8) return load_once8(p);
  else return load_once4(p);
}

// A vector of x a thread
template <typename V>
__device__ __forceinline__ void scatter_flat(long long block, const Sources& s, int vectors, const FastDiv& by_vectors, const V* x, const int32_t* slot,
                                             V* rows) {
  const FlatPlace p = flat_place(block, vectors, by_vectors);
  if (p.at >= (long long)s.tokens * vectors) return;
  const V v = load_vec<V>(x + p.at);
  const long long first = s.first(p.token);
  const int32_t* own = slot + (long long)p.token * s.k;
#pragma unroll 4
  for (int j = 0; j < s.k; ++j) {
    const unsigned to = (unsigned)__ldg(own + j);
    if (to < s.rows()) rows[(first + MS_AT((int)to, (int)s.rows())) * vectors + p.i] = v;
  }
}

// EACH times 32 vectors of a token a warp; a CTA is a box of warps: y the parts of a row that it has, z tokens side by side. Rows of more parts take several
// CTAs (`blocks`), next to one another.
constexpr int SCATTER_WARPS = FLAT_THREADS / 32;

template <typename V, int EACH>
__device__ __forceinline__ void scatter_rows(unsigned block, int blocks, const Sources& s, int vectors, const V* x, const int32_t* slot, V* rows) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, parts = (vectors + 32 * EACH - 1) / (32 * EACH);
  const int y = (parts + blocks - 1) / blocks, z = SCATTER_WARPS / y, of_token = warp / y;
  const unsigned set = blocks == 1 ? block : block / (unsigned)blocks, token = set * z + of_token;
  const int part = (int)(block - set * blocks) * y + warp - of_token * y;
  if (of_token >= z || token >= s.tokens) return;
  V v[EACH];
#pragma unroll
  for (int a = 0; a < EACH; ++a) {
    const int i = (part * EACH + a) * 32 + lane;
    if (i < vectors) v[a] = load_vec<V>(x + (size_t)token * vectors + i);
  }
  const unsigned own = lane < s.k ? (unsigned)slot[(long long)token * s.k + lane] : ~0u;
  const long long first = s.first(token);
#pragma unroll 4
  for (int j = 0; j < s.k; ++j) {
    const unsigned to = __shfl_sync(FULL, own, j);
    if (to >= s.rows()) continue;
#pragma unroll
    for (int a = 0; a < EACH; ++a) {
      const int i = (part * EACH + a) * 32 + lane;
      if (i < vectors) rows[(first + MS_AT((int)to, (int)s.rows())) * vectors + i] = v[a];
    }
  }
}

// The last CTAs have the scales, the others the tokens; EACH = 0: vectors of any token side by side
template <typename V, int EACH>
__global__ void __launch_bounds__(FLAT_THREADS) scatter_kernel(Sources s, unsigned ctas, int blocks, int vectors, FastDiv by_vectors, int scales,
                                                               FastDiv by_scales, const V* __restrict__ x, const float* __restrict__ scale,
                                                               const int32_t* __restrict__ slot, V* __restrict__ rows,
                                                               float* __restrict__ row_scale) {
  if (blockIdx.x >= ctas)
    scatter_flat<unsigned>(blockIdx.x - ctas, s, scales, by_scales, reinterpret_cast<const unsigned*>(scale), slot, reinterpret_cast<unsigned*>(row_scale));
  else if constexpr (EACH == 0) scatter_flat<V>(blockIdx.x, s, vectors, by_vectors, x, slot, rows);
  else scatter_rows<V, EACH>(blockIdx.x, blocks, s, vectors, x, slot, rows);
}

// whether there are so few warps that they should rather have less each (16 tokens of 4096 in bfloat16, 8 choices: 2.2 us with one vector a lane, 2.8 with four; the same
// at 500 warps of four; 592 tokens 7.5 and 7.3, of 7168 10.9 and 12.4 with 8 choices, 5.1 and 4.7 with 2)
static bool few_warps(long long warps) { return warps < 8LL * sm_count(); }

cudaError_t run_tokens_to_rows(int G, int T, int k, int row_bytes, int scales, const void* x, const float* scale, const int32_t* slot,
                               void* rows, float* row_scale, cudaStream_t stream) {
  const Sources s{(unsigned)G * T, T, k};
  const auto with = [&](auto vec, auto each) {
    using V = decltype(vec);
    constexpr int EACH = decltype(each)::value;
    const int vectors = row_bytes / (int)sizeof(V);
    int blocks = 1;
    long long ctas;
    if constexpr (EACH == 0) {
      ctas = flat_ctas((long long)s.tokens * vectors, 1);
    } else {
      const int parts = (vectors + 32 * EACH - 1) / (32 * EACH);
      blocks = (parts + SCATTER_WARPS - 1) / SCATTER_WARPS;
      const int z = SCATTER_WARPS / ((parts + blocks - 1) / blocks);
      ctas = ((long long)s.tokens + z - 1) / z * blocks;
    }
    return launch(scatter_kernel<V, EACH>, dim3((unsigned)(ctas + flat_ctas((long long)s.tokens * scales, 1))), dim3(FLAT_THREADS), 0, false, stream, s,
                  (unsigned)ctas, blocks, vectors, make_fastdiv(vectors), scales, make_fastdiv(scales > 0 ? scales : 1), static_cast<const V*>(x), scale,
                  slot, static_cast<V*>(rows), row_scale);
  };
  const auto with_each = [&](auto vec) {
    const int vectors = row_bytes / (int)sizeof(vec);
    if (vectors < 32) return with(vec, std::integral_constant<int, 0>());
    if (few_warps((long long)s.tokens * ((vectors + 127) / 128))) return with(vec, std::integral_constant<int, 1>());
    return with(vec, std::integral_constant<int, 4>());
  };
  return row_bytes % 16 == 0 ? with_each(uint4()) : with_each(uint2());
}

// ROWS rows at a time of EACH vectors a thread
template <typename T, int ROWS, int EACH>
__global__ void __launch_bounds__(FLAT_THREADS) gather_kernel(Sources s, int vectors, FastDiv by_vectors, const uint4* __restrict__ rows,
                                                              const int32_t* __restrict__ slot, const float* __restrict__ weights, const uint4* add,
                                                              uint4* y) {
  constexpr int COUNT = Vec<T>::COUNT;
  const long long all = (long long)s.tokens * vectors;
  FlatPlace p[EACH];
  float sum[EACH][COUNT];
#pragma unroll
  for (int a = 0; a < EACH; ++a) {
    p[a] = flat_place((long long)blockIdx.x * EACH + a, vectors, by_vectors);
    if (p[a].at >= all) p[a].token = 0u;
#pragma unroll
    for (int e = 0; e < COUNT; ++e) sum[a][e] = 0.0f;
    if (add != nullptr && p[a].at < all) Vec<T>::unpack(load_once(add + p[a].at), sum[a]);
  }
  for (int j0 = 0; j0 < s.k; j0 += ROWS) {
    uint4 v[EACH][ROWS];
    unsigned from[EACH][ROWS];
#pragma unroll
    for (int a = 0; a < EACH; ++a)
#pragma unroll
      for (int q = 0; q < ROWS; ++q)
        from[a][q] = j0 + q < s.k && p[a].at < all ? (unsigned)__ldg(slot + (long long)p[a].token * s.k + j0 + q) : ~0u;
#pragma unroll
    for (int a = 0; a < EACH; ++a)
#pragma unroll
      for (int q = 0; q < ROWS; ++q)
        if (from[a][q] < s.rows()) v[a][q] = load_once(rows + (s.first(p[a].token) + MS_AT((int)from[a][q], (int)s.rows())) * vectors + p[a].i);
#pragma unroll
    for (int a = 0; a < EACH; ++a)
#pragma unroll
      for (int q = 0; q < ROWS; ++q) {
        if (from[a][q] >= s.rows()) continue;
        const float w = weights != nullptr ? __ldg(weights + (long long)p[a].token * s.k + j0 + q) : 1.0f;
        float f[COUNT];
        Vec<T>::unpack(v[a][q], f);
#pragma unroll
        for (int e = 0; e < COUNT; ++e) sum[a][e] = fmaf(w, f[e], sum[a][e]);
      }
  }
#pragma unroll
  for (int a = 0; a < EACH; ++a)
    if (p[a].at < all) y[p[a].at] = Vec<T>::pack(sum[a]);
}

cudaError_t run_rows_to_tokens(int G, int T, int k, int D, int dtype, const void* rows, const int32_t* slot, const float* weights,
                               const void* add, void* y, cudaStream_t stream) {
  const Sources s{(unsigned)G * T, T, k};
  return with_type(dtype, [&](auto type) {
    using V = decltype(type);
    const int vectors = D / Vec<V>::COUNT;
    const long long all = (long long)s.tokens * vectors;
    const auto with = [&](auto kern, int each) {
      return launch(kern, dim3((unsigned)flat_ctas(all, each)), dim3(FLAT_THREADS), 0, false, stream, s, vectors, make_fastdiv(vectors),
                    static_cast<const uint4*>(rows), slot, weights, static_cast<const uint4*>(add), static_cast<uint4*>(y));
    };
    // Few threads have all of their rows on their way at once (4096 in bfloat16, 8 choices: 16 tokens 2.8 us, 3.1 with four rows at a time; 296 tokens, four times the limit, 4.3
    // and 4.6; 8191 tokens 111 and 106); one or two rows a token need several vectors a thread (65536 tokens of 2048: one choice 154 us with four vectors, 179 with one; two
    // choices 180 with two, 213 with four, 209 with one).
    if (all < 256LL * sm_count()) return with(gather_kernel<V, 8, 1>, 1);
    if (k == 1) return with(gather_kernel<V, 1, 4>, 4);
    if (k == 2) return with(gather_kernel<V, 2, 2>, 2);
    return with(gather_kernel<V, 4, 1>, 1);
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

// Row of a choice, counted from the first source; negative: not sent
__device__ __forceinline__ long long row_of(const int32_t* slot, unsigned token, int k, int per, int j, bool wanted) {
  if (!wanted) return -1;
  const int at = slot[(long long)token * k + j], rows = per * k;
  return (unsigned)at < (unsigned)rows ? (long long)(token / (unsigned)per) * rows + MS_AT(at, rows) : -1;
}

// Gradients of the weighted sum: drows[slot] = w dy[t], dw = <dy[t], rows[slot]>. The warps of a token (z: tokens side by side) go over its vectors, VECTORS a lane
// and ROWS rows at a time. drows may be rows itself: a vector is read by the thread that writes it, before it does.
// (64 registers, for two CTAs of 512: 36 bytes of them spilled in 16 bits with two rows of two vectors.)
template <typename T, int ROWS, int VECTORS>
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
    for (int i0 = 32 * VECTORS * warp + lane; i0 - lane < vectors; i0 += 32 * VECTORS * warps) {
      uint4 v[VECTORS][ROWS], d[VECTORS];
#pragma unroll
      for (int a = 0; a < VECTORS; ++a) {
        const int i = i0 + 32 * a;
#pragma unroll
        for (int q = 0; q < ROWS; ++q)
          if (at[q] >= 0 && i < vectors) v[a][q] = load_once(rows + at[q] * vectors + i);
        d[a] = active && i < vectors ? dy[(size_t)token * vectors + i] : make_uint4(0u, 0u, 0u, 0u);
      }
#pragma unroll
      for (int a = 0; a < VECTORS; ++a) {
        const int i = i0 + 32 * a;
        float g[COUNT];
        Vec<T>::unpack(d[a], g);
#pragma unroll
        for (int q = 0; q < ROWS; ++q) {
          const float w = __shfl_sync(FULL, weight, (j0 + q) & 31);
          if (at[q] < 0 || i >= vectors) continue;
          float f[COUNT];
          Vec<T>::unpack(v[a][q], f);
#pragma unroll
          for (int e = 0; e < COUNT; ++e) {
            sum[q] = fmaf(g[e], f[e], sum[q]);
            f[e] = g[e] * w;
          }
          drows[at[q] * vectors + i] = Vec<T>::pack(f);
        }
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
    const int vectors = D / Vec<V>::COUNT;
    const auto with = [&](auto kern, int warps, int z) {
      return launch(kern, dim3((tokens + z - 1) / z), dim3(32, warps, z), 0, false, stream, tokens, T, k, vectors,
                    static_cast<const uint4*>(dy), static_cast<const uint4*>(rows), slot, weights, static_cast<uint4*>(drows), dweights);
    };
    const int all = (vectors + 31) / 32;                        // parts of a row that a warp takes at a time
    // Below 16 parts an SM all rows at once (4096, 8 choices: 16 tokens 4.1 us, 4.5 with four rows at a time; 148 tokens, the limit, 4.5 and 4.9; 222 tokens 7.5 and 6.4.
    // With two choices 3.4, and 2.9 with two rows at a time.)
    const long long enough = 16LL * sm_count();
    if (tokens * (long long)all < enough) return with(gather_backward_kernel<V, 8, 1>, all < 16 ? all : 16, 1);
    // A token's warps have a few parts each, so that what a token costs once is spread over them (bfloat16. 8 rows of 4096, 8191 tokens: 1 warp 202 us, 2 190, 4 and 8 182;
    // 4 rows of 2048, 16384 tokens: 1 warp 102 us, 2 97, 4 98, 8 116; 8 rows of 264, 60000 tokens: 1 warp 130 us, 2 142; 1 row of 2048, 32768 tokens: 1 warp 66, 2 72),
    // unless the tokens are few
    int warps = all / (k > 4 ? 2 : 4);
    warps = warps < 1 ? 1 : warps > 4 ? 4 : warps;
    while (2 * warps <= 16 && 2 * warps <= all && tokens * (long long)warps < enough) warps *= 2;
    const int z = warps < 4 ? 4 / warps : 1;
    return k <= 2 ? with(gather_backward_kernel<V, 2, 2>, warps, z) : with(gather_backward_kernel<V, 4, 1>, warps, z);
  });
}

// 8-bit rows to the type: y = q scale, a scale for every 2^shift vectors of a row. A thread has as many values as 16 bytes of the type hold, a few times.
template <typename T, int EACH>
__global__ void __launch_bounds__(FLAT_THREADS) widen_kernel(long long all, int vectors, FastDiv by_vectors, int shift, int scales,
                                                             const uint8_t* __restrict__ q, const float* __restrict__ scale, uint4* __restrict__ y) {
  constexpr int COUNT = Vec<T>::COUNT;
  using Bytes = std::conditional_t<COUNT == 8, uint2, unsigned>;
  FlatPlace p[EACH];
  Bytes v[EACH];
  float s[EACH];
#pragma unroll
  for (int a = 0; a < EACH; ++a) {
    p[a] = flat_place((long long)blockIdx.x * EACH + a, vectors, by_vectors);
    if (p[a].at >= all) continue;
    v[a] = load_vec<Bytes>(q + p[a].at * COUNT);
    s[a] = __ldg(scale + (size_t)p[a].token * scales + (p[a].i >> shift));
  }
#pragma unroll
  for (int a = 0; a < EACH; ++a) {
    if (p[a].at >= all) return;
    const unsigned* words = reinterpret_cast<const unsigned*>(&v[a]);
    float f[COUNT];
#pragma unroll
    for (int e = 0; e < COUNT; e += 2) {
      const __half2_raw both = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(words[e / 4] >> (8 * (e & 2))), __NV_E4M3);
      const float2 wide = __half22float2(*reinterpret_cast<const __half2*>(&both));
      f[e] = wide.x * s[a];
      f[e + 1] = wide.y * s[a];
    }
    y[p[a].at] = Vec<T>::pack(f);
  }
}

cudaError_t run_rows_widen(int R, int D, int group, int dtype, const uint8_t* q, const float* scale, void* y, cudaStream_t stream) {
  return with_type(dtype, [&](auto type) {
    using V = decltype(type);
    constexpr int EACH = 2;
    int shift = 0;
    while (Vec<V>::COUNT << shift < group) ++shift;
    const int vectors = D / Vec<V>::COUNT;
    const long long all = (long long)R * vectors;
    return launch(widen_kernel<V, EACH>, dim3((unsigned)flat_ctas(all, EACH)), dim3(FLAT_THREADS), 0, false, stream, all, vectors,
                  make_fastdiv(vectors), shift, (D + group - 1) / group, q, scale, static_cast<uint4*>(y));
  });
}

}  // namespace moesched
