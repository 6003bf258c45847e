// The router's choice: the k experts of a token with the greatest score, and their weights.
//
// Scores are the softmax or the logistic function of the token's logits l. Without a bias the order of the scores is that of the logits,
// and those are compared as they are. With a bias b, score + b decides, and is compared as it is in 64 bits: it is computed in 32
// first, with a bound of its error, and again in 64 where two of the k + 1 greatest are nearer than their bounds. Equal ones: the lowest expert.
// Weights come from the logits of the chosen alone where they are normalised:
//   softmax   w = e^(l - m) / sum e^(l - m),  m the greatest of them
//   logistic  w = t / sum t,  t = e^(l - m) / (1 + e^l),  m = min(0, the greatest): it has no common factor left that could underflow
// One warp has a token, lane i the experts i, i + 32, ...; the greatest is found with two reductions over the warp (value, then lowest expert).
#include "token.cuh"

namespace moesched {

constexpr int CHOOSE_WARPS = 8;

// Numbers in an order that whole numbers have; 0 below all of them, for an expert that cannot be chosen
__device__ __forceinline__ unsigned ordered(float v) {
  if (!(v > -INFINITY)) return 0u;                               // (NaN too)
  const unsigned u = __float_as_uint(v + 0.0f);                  // (-0 and 0 are equal)
  return (u & 0x80000000u) != 0u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(unsigned u) { return __uint_as_float((u & 0x80000000u) != 0u ? u ^ 0x80000000u : ~u); }
__device__ __forceinline__ unsigned long long ordered(double v) {
  if (!(v > -INFINITY)) return 0ull;
  const unsigned long long u = (unsigned long long)__double_as_longlong(v + 0.0);
  return (u >> 63) != 0ull ? ~u : u | 0x8000000000000000ull;
}
__device__ __forceinline__ unsigned warp_most(unsigned v) { return __reduce_max_sync(FULL, v); }
__device__ __forceinline__ unsigned long long warp_most(unsigned long long v) {
  const unsigned hi = __reduce_max_sync(FULL, (unsigned)(v >> 32));
  const unsigned lo = __reduce_max_sync(FULL, (unsigned)(v >> 32) == hi ? (unsigned)v : 0u);
  return (unsigned long long)hi << 32 | lo;
}
__device__ __forceinline__ float warp_most(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(FULL, v, o));
  return v;
}

// Lane i gets the expert of the i-th greatest key, -1 where no key is left; `between(a, b)` sees each key and the next, as many as `count` + 1
template <int J, typename Key, typename Between>
__device__ __forceinline__ int greatest(Key (&key)[J], int count, Between between) {
  const int lane = threadIdx.x & 31;
  int mine = -1;
  Key before = 0;
  for (int r = 0;; ++r) {
    Key best = 0;
    int at = 0;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      at = key[j] > best ? j : at;
      best = key[j] > best ? key[j] : best;
    }
    const Key most = warp_most(best);
    if (r > 0) between(before, most);
    if (r == count || most == 0) break;
    const int expert = (int)__reduce_min_sync(FULL, best == most ? 32u * at + lane : 0xffffffffu);
    if (lane == r) mine = expert;
#pragma unroll
    for (int j = 0; j < J; ++j) key[j] = 32 * j + lane == expert ? Key(0) : key[j];
    before = most;
  }
  return mine;
}

template <typename T, int J>
__device__ __forceinline__ void load_logits(const T* logits, int E, float (&l)[J]) {
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int e = 32 * j + (threadIdx.x & 31);
    l[j] = e < E ? to_float(logits[e]) : -INFINITY;
  }
}

// greatest logit of the row, and the sum of e^(l - m); the sum of a row without a logit is 0
template <int J>
__device__ __forceinline__ void softmax_of(const float (&l)[J], float& m, float& sum) {
  m = l[0];
#pragma unroll
  for (int j = 1; j < J; ++j) m = fmaxf(m, l[j]);
  m = warp_most(m);
  sum = 0.0f;
  if (m == -INFINITY) return;
#pragma unroll
  for (int j = 0; j < J; ++j) sum += expf(l[j] - m);
  sum = warp_sum(sum);
}

__device__ __noinline__ double exp64(double v) { return exp(v); }

// Scores and choices in 64 bits
template <int J, int SCORE>
__device__ __noinline__ int choose64(const float (&l)[J], const float* bias, int E, int k, float top) {
  const int lane = threadIdx.x & 31;
  double sum = 0.0;
  unsigned long long key[J];
  if constexpr (SCORE == MOESCHED_SCORE_SOFTMAX) {
#pragma unroll
    for (int j = 0; j < J; ++j) sum += exp64((double)l[j] - (double)top);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(FULL, sum, o);
  }
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int e = 32 * j + lane;
    key[j] = 0ull;
    if (e >= E || !(l[j] > -INFINITY)) continue;
    const double s = SCORE == MOESCHED_SCORE_SOFTMAX ? exp64((double)l[j] - (double)top) / sum : 1.0 / (1.0 + exp64(-(double)l[j]));
    key[j] = ordered(s + (double)bias[e]);
  }
  return greatest(key, k, [](unsigned long long, unsigned long long) {});
}

template <typename T, int J, int SCORE>
__global__ void __launch_bounds__(32 * CHOOSE_WARPS) choose_kernel(int rows, int E, int k, int normalise, float factor,
                                                                   const T* __restrict__ logits, const float* __restrict__ bias,
                                                                   int32_t* __restrict__ experts, float* __restrict__ weights) {
  constexpr bool SOFTMAX = SCORE == MOESCHED_SCORE_SOFTMAX;
  const int lane = threadIdx.x & 31;
  const long long row = (long long)blockIdx.x * CHOOSE_WARPS + (threadIdx.x >> 5);
  if (row >= rows) return;
  const T* own = logits + row * E;
  float l[J], top = 0.0f, sum = 0.0f;
  load_logits(own, E, l);
  bool lost = false;
#pragma unroll
  for (int j = 0; j < J; ++j) lost |= isnan(l[j]);
  lost = __any_sync(FULL, lost);
  if (SOFTMAX && (bias != nullptr || !normalise)) softmax_of(l, top, sum);
  unsigned key[J];
  int expert;
  if (bias == nullptr) {
#pragma unroll
    for (int j = 0; j < J; ++j) key[j] = ordered(l[j]);
    expert = greatest(key, k, [](unsigned, unsigned) {});
  } else {
    bool near = false;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int e = 32 * j + lane;
      const float s = SOFTMAX ? expf(l[j] - top) / sum : 1.0f / (1.0f + expf(-l[j]));
      key[j] = e < E && l[j] > -INFINITY ? ordered(s + bias[e]) : 0u;
    }
    // A score is at most 1 and off by 2^-18 at most (its exponential by 2 steps of 2^-23 and by that of its argument, which is x 2^-24 with x e^-x < 0.4;
    // the sum of up to 32 on a lane and over 32 lanes by 37 half steps; the quotient), the sum with the bias by half a step of its own.
    expert = greatest(key, k, [&](unsigned a, unsigned b) {
      if (b == 0u) return;
      const float u = unordered(a), v = unordered(b);
      near |= !(u - v > 0x1p-17f + 0x1p-23f * (fabsf(u) + fabsf(v)));
    });
    if (near) expert = choose64<J, SCORE>(l, bias, E, k, top);
  }
  const bool there = expert >= 0;
  const float mine = there ? to_float(own[expert]) : -INFINITY;
  float w;
  if (normalise) {
    const float most = warp_most(mine), m = SOFTMAX ? most : fminf(most, 0.0f);
    if (SOFTMAX) w = expf(mine - m);
    else w = mine > 0.0f ? 1.0f / (1.0f + expf(-mine)) : expf(mine - m) / (1.0f + expf(mine));
    w = there ? w : 0.0f;
    w = w / warp_sum(w);
  } else {
    w = SOFTMAX ? expf(mine - top) / sum : 1.0f / (1.0f + expf(-mine));
  }
  if (lane < k) {
    experts[row * k + lane] = expert;
    weights[row * k + lane] = lost ? NAN : there ? w * factor : 0.0f;
  }
}

// Gradients of the logits, from a = factor * dw:
//   softmax             p (a [chosen] - sum a p)      over all experts
//   softmax, normalised q (a - sum a q)               over the chosen, 0 for the others
//   logistic            a s (1 - s);  normalised  q (a - sum a q) (1 - s)
template <typename T, int J, int SCORE>
__global__ void __launch_bounds__(32 * CHOOSE_WARPS) choose_backward_kernel(int rows, int E, int k, int normalise, float factor,
                                                                            const float* __restrict__ dweights,
                                                                            const T* __restrict__ logits,
                                                                            const int32_t* __restrict__ experts, T* dlogits) {
  constexpr bool SOFTMAX = SCORE == MOESCHED_SCORE_SOFTMAX;
  const int lane = threadIdx.x & 31;
  const long long row = (long long)blockIdx.x * CHOOSE_WARPS + (threadIdx.x >> 5);
  if (row >= rows) return;
  const T* own = logits + row * E;
  T* out = dlogits + row * E;
  int expert = lane < k ? experts[row * k + lane] : -1;
  if ((unsigned)expert >= (unsigned)E) expert = -1;
  const bool there = expert >= 0;
  const float mine = there ? to_float(own[expert]) : -INFINITY;
  const float a = there ? dweights[row * k + lane] * factor : 0.0f;
  float d, dot = 0.0f;
  if (normalise) {
    const float most = warp_most(mine), m = SOFTMAX ? most : fminf(most, 0.0f);
    float q;
    if (SOFTMAX) q = expf(mine - m);
    else q = mine > 0.0f ? 1.0f / (1.0f + expf(-mine)) : expf(mine - m) / (1.0f + expf(mine));
    q = there ? q : 0.0f;
    q = q / warp_sum(q);
    dot = warp_sum(there ? a * q : 0.0f);
    d = q * (a - dot);
    if (!SOFTMAX) d /= 1.0f + expf(mine);                        // 1 - s
  } else if (SOFTMAX) {
    float l[J], top, sum;
    load_logits(own, E, l);
    softmax_of(l, top, sum);
    const float p = there ? expf(mine - top) / sum : 0.0f;
    dot = warp_sum(a * p);
    d = p * (a - dot);
#pragma unroll
    for (int j = 0; j < J; ++j)
      if (32 * j + lane < E) put(out + 32 * j + lane, l[j] == -INFINITY ? 0.0f : expf(l[j] - top) / sum * -dot);
  } else {
    const float s = 1.0f / (1.0f + expf(-mine));
    d = a * s / (1.0f + expf(mine));
  }
  if (!SOFTMAX || normalise)
    for (int e = lane; e < E; e += 32) put(out + e, 0.0f);
  __syncwarp();                                                  // the chosen after all of them
  if (there) put(out + expert, d);
}

template <typename Call>
static cudaError_t with_experts(int E, Call call) {
  if (E <= 32) return call(std::integral_constant<int, 1>());
  if (E <= 64) return call(std::integral_constant<int, 2>());
  if (E <= 128) return call(std::integral_constant<int, 4>());
  if (E <= 256) return call(std::integral_constant<int, 8>());
  if (E <= 512) return call(std::integral_constant<int, 16>());
  return call(std::integral_constant<int, 32>());
}

cudaError_t run_choose(int rows, int E, int k, int dtype, int score, int normalise, float factor, const void* logits, const float* bias,
                       int32_t* experts, float* weights, cudaStream_t stream) {
  if (rows == 0) return cudaSuccess;
  return with_type(dtype, [&](auto type) {
    using T = decltype(type);
    return with_experts(E, [&](auto count) {
      constexpr int J = decltype(count)::value;
      const auto kern = score == MOESCHED_SCORE_SOFTMAX ? choose_kernel<T, J, MOESCHED_SCORE_SOFTMAX> : choose_kernel<T, J, MOESCHED_SCORE_SIGMOID>;
      return launch(kern, (rows + CHOOSE_WARPS - 1) / CHOOSE_WARPS, 32 * CHOOSE_WARPS, 0, stream, rows, E, k, normalise, factor,
                    static_cast<const T*>(logits), bias, experts, weights);
    });
  });
}

cudaError_t run_choose_backward(int rows, int E, int k, int dtype, int score, int normalise, float factor, const float* dweights,
                                const void* logits, const int32_t* experts, void* dlogits, cudaStream_t stream) {
  if (rows == 0) return cudaSuccess;
  return with_type(dtype, [&](auto type) {
    using T = decltype(type);
    return with_experts(E, [&](auto count) {
      constexpr int J = decltype(count)::value;
      const auto kern = score == MOESCHED_SCORE_SOFTMAX ? choose_backward_kernel<T, J, MOESCHED_SCORE_SOFTMAX>
                                                        : choose_backward_kernel<T, J, MOESCHED_SCORE_SIGMOID>;
      return launch(kern, (rows + CHOOSE_WARPS - 1) / CHOOSE_WARPS, 32 * CHOOSE_WARPS, 0, stream, rows, E, k, normalise, factor, dweights,
                    static_cast<const T*>(logits), experts, static_cast<T*>(dlogits));
    });
  });
}

}  // namespace moesched
