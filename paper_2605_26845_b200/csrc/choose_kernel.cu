// The router's choice: the k experts of a token with the greatest score, and their weights.
//
// Scores are the softmax or the logistic function of the token's logits l. Without a bias the order of the scores is that of the logits,
// and those are compared as they are. With a bias b, score + b decides, and is compared as it is in 64 bits: it is computed in 32
// first, with a bound of its error, and again in 64 where two of the k + 1 greatest are nearer than their bounds. Equal ones: the lowest expert.
// (All that is near enough to be chosen is gathered, so that only those scores are computed again, unless they are more than 32. The bound of the error is one for all scores, and
// those of a softmax that is nearly even lie within it: with a bias of 0 and logits of a spread of 1.5, 0.5, 0.1 and 0.02, 16384 x 256 take 14.7, 17.1, 24.3 and 27.0 us, and
// 8192 x 1024 47.7, 70.1, 72.7 and 173.4, where at 0.02 nearly every token has more than 32. Logistic: 11.7 to 12.8 and 43 to 45.)
// Weights come from the logits of the chosen alone where they are normalised:
//   softmax   w = e^(l - m) / sum e^(l - m),  m the greatest of them
//   logistic  w = t / sum t,  t = e^(l - m) / (1 + e^l),  m = min(0, the greatest): it has no common factor left that could underflow
// One warp has a token, lane i the experts i J .. i J + J - 1. It finds a bound that no wanted key is below, gathers what is left (10 of 256 usually) one a
// lane, and each counts the keys before its own. Instructions bound it: 8 of 256 experts for 16384 tokens take 7.9 us, 387 instructions a token, 73 % of what can be issued
// (the bytes alone 2.8 us); with a bias 11.5 (logistic) and 14.1 (softmax, which spills 20 bytes for its five CTAs an SM); 8 of 1024 for 8192 tokens 14.3, with a bias 43; the greatest of all keys k times over, as more than 32 candidates have it, 16.3. The gradient takes 5.5 us, bound by its
// stores and the way from a choice to its logit.
#include <cfloat>

#include "token.cuh"

namespace moesched {

constexpr int CHOOSE_WARPS = 8;

// Numbers in an order that whole numbers have; 0 below all of them, for an expert that cannot be chosen
__device__ __forceinline__ unsigned ordered(float v) {
  if (!(v > -INFINITY)) return 0u;                               // (NaN too)
  const unsigned u = __float_as_uint(v + 0.0f);                  // (-0 and 0 are equal)
  return (u & 0x80000000u) != 0u ? ~u : u | 0x80000000u;
}
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
__device__ __forceinline__ float warp_most(float v) {            // NaN is none
  asm volatile("redux.sync.max.f32 %0, %0, 0xffffffff;" : "+f"(v));
  return v;
}
__device__ __forceinline__ float warp_most_or_nan(float v) {
  asm volatile("redux.sync.max.NaN.f32 %0, %0, 0xffffffff;" : "+f"(v));
  return v;
}

// Lane i gets the expert of the i-th greatest key, -1 where no key is left, `count` of them in falling order
template <int J, typename Key>
__device__ __forceinline__ int greatest(Key (&key)[J], int count) {
  const int lane = threadIdx.x & 31;
  int mine = -1;
  for (int r = 0; r < count; ++r) {
    Key best = key[0];
    int at = 0;
#pragma unroll
    for (int j = 1; j < J; ++j) {
      at = key[j] > best ? j : at;
      best = key[j] > best ? key[j] : best;
    }
    const Key most = warp_most(best);
    if (most == 0) break;
    const int expert = (int)__reduce_min_sync(FULL, best == most ? (unsigned)(lane * J + at) : 0xffffffffu);
    if (lane == r) mine = expert;
#pragma unroll
    for (int j = 0; j < J; ++j) key[j] = lane * J + j == expert ? Key(0) : key[j];
  }
  return mine;
}

// The keys that may be among the `count` greatest, in falling order, the lowest expert first among equal ones: lane i gets the i-th. The count-th greatest of
// the lanes' own greatest keys has `count` keys at or above it, so that nothing below it is wanted; spare(key) is the lowest key that has to be looked at
// all the same. Returns how many there are: with more than 32, nothing else holds. -infinity and NaN are no keys. best: the lane's greatest; list: [64], of the
// warp.
template <int J, typename Spare>
__device__ __forceinline__ int candidates(const float (&key)[J], float best, int count, uint2* list, Spare spare, float& own, int& expert) {
  const int lane = threadIdx.x & 31;
  float bound = -INFINITY;
  for (int r = 0; r < count; ++r) {                             // (equal ones go together: the bound is only lower for it)
    bound = warp_most(best);
    best = best == bound ? -INFINITY : best;
  }
  bound = fmaxf(spare(bound), -FLT_MAX);
  int at = 0, found = 0;
  if constexpr (J <= 4) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const unsigned who = __ballot_sync(FULL, key[j] >= bound);
      at += __popc(who & ((1u << lane) - 1u));
      found += __popc(who);
    }
  } else {
    int mine = 0;
#pragma unroll
    for (int j = 0; j < J; ++j) mine += key[j] >= bound;
    at = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(FULL, at, o);
      if (lane >= o) at += v;
    }
    found = __shfl_sync(FULL, at, 31);
    at -= mine;
  }
  if (found > 32) {
    own = -INFINITY;
    expert = -1;
    return found;
  }
#pragma unroll
  for (int j = 0; j < J; ++j)
    if (key[j] >= bound) list[MS_AT(at++, 32)] = make_uint2(__float_as_uint(key[j]), lane * J + j);
  __syncwarp();
  // up to 16 keys: two lanes for each, which count among one half of them
  const bool two_each = found <= 16;
  const int which = two_each ? lane & 15 : lane, half = (found + 1) / 2, from = two_each && lane >= 16 ? half : 0, steps = two_each ? half : found;
  const uint2 entry = which < found ? list[which] : make_uint2(0xff800000u, 0u);
  const unsigned mine = ordered(__uint_as_float(entry.x));
  int place = 0;
#pragma unroll 2
  for (int i = 0; i < steps; ++i) {
    const unsigned other = __shfl_sync(FULL, mine, from + i);
    place += other + (from + i < which) > mine;                 // (no key is the greatest number)
  }
  if (two_each) place += __shfl_xor_sync(FULL, place, 16);
  if (lane < found) list[32 + MS_AT(place, 32)] = entry;
  __syncwarp();
  const uint2 sorted = lane < found ? list[32 + lane] : make_uint2(0xff800000u, 0xffffffffu);
  own = __uint_as_float(sorted.x);
  expert = (int)sorted.y;
  return found;
}

// How near two scores with their biases, in 32 bits, may be to one another without their order being known. A score is off by 2^-18 at most, 32 steps of 2^-23. Softmax, of
// the greatest logit less x: its exponential by 2 + 1.17 x relatively and half of x for its argument, which e^-x leaves 2.2 of; the sum's exponentials by 2 and half of x, 4.3 in the
// mean of their sizes where 1023 of them are the same, and its 36 additions by 18; the reciprocal and the product by 2.5. Logistic: less than 4. The sum with the bias is off by half a step of its
// own.
__device__ __forceinline__ float apart(float u, float v) { return 0x1p-17f + 0x1p-23f * (fabsf(u) + fabsf(v)); }

// The lane's logits (or biases), -infinity where there is no expert. wide: as many as 16 bytes hold at a time
template <typename T, int J>
__device__ __forceinline__ void load_logits(const T* logits, int E, bool wide, float (&l)[J]) {
  constexpr int COUNT = Vec<T>::COUNT;
  constexpr unsigned NONE = sizeof(T) == 4 ? 0xff800000u : std::is_same_v<T, __half> ? 0xfc00fc00u : 0xff80ff80u;
  const int first = (threadIdx.x & 31) * J;
  if (J % COUNT == 0 && wide) {
#pragma unroll
    for (int j = 0; j < J; j += COUNT) {
      float f[COUNT];
      uint4 v = make_uint4(NONE, NONE, NONE, NONE);
      if (first + j < E) v = __ldg(reinterpret_cast<const uint4*>(logits + first + j));
      Vec<T>::unpack(v, f);
#pragma unroll
      for (int q = 0; q < COUNT; ++q)
        if (j + q < J) l[j + q] = f[q];
    }
  } else {
#pragma unroll
    for (int j = 0; j < J; ++j) l[j] = first + j < E ? to_float(logits[first + j]) : -INFINITY;
  }
}

// Scores that are compared and no more: e^v with an error that grows with v, for which `apart` allows. (The quotient is of a number between 1 and 2^126, or 0.)
__device__ __forceinline__ float rough_exponential(float v) { return __expf(v); }
__device__ __forceinline__ float rough_logistic(float v) { return __fdividef(1.0f, 1.0f + rough_exponential(-v)); }

// What is given out: exponentials of 32 bits, and quotients whose remainder is put back, which rounds all but one in 500 000 as the division does and spares its way
// around numbers that do not come here: b is between 1/2 and 2^11, or a NaN. (16384 x 256 7.9 us; with divisions 8.6, with quotients and exponentials as above 7.7.)
__device__ __forceinline__ float quotient(float a, float b) {
  const float r = __fdividef(1.0f, b), q = a * r;
  return fmaf(fmaf(-q, b, a), r, q);
}
// 1 / (1 + e^-v), and its slope, from e^-|v|, which neither overflows nor loses what is small
__device__ __forceinline__ float logistic(float v) {
  const float e = expf(-fabsf(v));
  return quotient(v > 0.0f ? 1.0f : e, 1.0f + e);
}
__device__ __forceinline__ float logistic_slope(float v) {
  const float e = expf(-fabsf(v)), sum = 1.0f + e;
  return quotient(e, sum * sum);
}

template <int J>
__device__ __forceinline__ float most_of(const float (&v)[J]) {
  float m = fmaxf(v[0], -INFINITY);
#pragma unroll
  for (int j = 1; j < J; ++j) m = fmaxf(m, v[j]);
  return m;
}

// greatest logit of the row, and the sum of e^(l - m); the sum of a row without a logit is 0
template <int J>
__device__ __forceinline__ void softmax_of(const float (&l)[J], float& m, float& sum) {
  m = warp_most(most_of(l));
  sum = 0.0f;
  if (m == -INFINITY) return;
#pragma unroll
  for (int j = 0; j < J; ++j) sum += expf(l[j] - m);
  sum = warp_sum(sum);
}

// Normalised scores of the chosen, a lane's from its logit: see above
template <bool SOFTMAX>
__device__ __forceinline__ float normalised(float l, bool there) {
  const float most = warp_most(l), m = SOFTMAX ? most : fminf(most, 0.0f);
  float w = SOFTMAX ? expf(l - m) : quotient(expf(fminf(l, 0.0f) - m), 1.0f + expf(-fabsf(l)));
  w = there ? w : 0.0f;
  const float sum = warp_sum(w);
  return there ? quotient(w, sum) : 0.0f;
}

__device__ __noinline__ double exp64(double v) { return exp(v); }

template <int J>
__device__ __noinline__ double softmax_sum64(const float (&l)[J], float top) {
  double sum = 0.0;
#pragma unroll
  for (int j = 0; j < J; ++j) sum += exp64((double)l[j] - (double)top);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(FULL, sum, o);
  return sum;
}
template <int SCORE>
__device__ __forceinline__ unsigned long long key64(float l, float bias, float top, double sum) {
  if (!(l > -INFINITY)) return 0ull;
  return ordered((SCORE == MOESCHED_SCORE_SOFTMAX ? exp64((double)l - (double)top) / sum : 1.0 / (1.0 + exp64(-(double)l))) + (double)bias);
}

// The order of up to 32 experts, one a lane, by their scores in 64 bits: lane i gets the i-th
template <int SCORE>
__device__ __noinline__ int order64(float l, float bias, float top, double sum, int expert, int found, uint2* list) {
  const int lane = threadIdx.x & 31;
  const unsigned long long mine = lane < found ? key64<SCORE>(l, bias, top, sum) : 0ull;
  int place = 0;
  for (int i = 0; i < found; ++i) {
    const unsigned long long other = __shfl_sync(FULL, mine, i);
    const int its = __shfl_sync(FULL, expert, i);
    place += other > mine || (other == mine && its < expert);
  }
  __syncwarp();
  if (lane < found) list[MS_AT(place, 32)].y = (unsigned)expert;
  __syncwarp();
  return lane < found ? (int)list[lane].y : -1;
}

// All scores and the choice in 64 bits
template <int J, int SCORE>
__device__ __noinline__ int choose64(const float (&l)[J], const float* bias, int E, int k, float top, double sum) {
  const int first = (threadIdx.x & 31) * J;
  unsigned long long key[J];
#pragma unroll
  for (int j = 0; j < J; ++j) key[j] = first + j < E ? key64<SCORE>(l[j], bias[first + j], top, sum) : 0ull;
  return greatest(key, k);
}

// The choice of a token whose softmax is NaN: by its logits, as without a bias, of the experts that the bias leaves
template <int J>
__device__ __noinline__ int choose_lost(const float (&l)[J], const float* bias, int E, int k) {
  const int first = (threadIdx.x & 31) * J;
  unsigned key[J];
#pragma unroll
  for (int j = 0; j < J; ++j) key[j] = first + j < E && bias[first + j] > -INFINITY ? ordered(l[j]) : 0u;
  return greatest(key, k);
}

template <typename T, int J, int SCORE, bool BIAS>
__global__ void __launch_bounds__(32 * CHOOSE_WARPS, J <= 8 ? 5 : 1) choose_kernel(int rows, int E, int k, int normalise, int wide, float factor,
                                                                   const T* __restrict__ logits, const float* __restrict__ bias,
                                                                   int32_t* __restrict__ experts, float* __restrict__ weights) {
  constexpr bool SOFTMAX = SCORE == MOESCHED_SCORE_SOFTMAX;
  __shared__ uint2 lists[CHOOSE_WARPS][64];
  uint2* list = lists[threadIdx.x >> 5];
  const int lane = threadIdx.x & 31;
  const long long row = (long long)blockIdx.x * CHOOSE_WARPS + (threadIdx.x >> 5);
  if (row >= rows) return;
  const T* own = logits + row * E;
  float l[J], top = 0.0f, sum = 0.0f, best = 0.0f;
  load_logits(own, E, wide != 0, l);
  best = l[0];
#pragma unroll
  for (int j = 1; j < J; ++j) asm("max.NaN.f32 %0, %0, %1;" : "+f"(best) : "f"(l[j]));
  const float most = warp_most_or_nan(best);
  const bool lost = SOFTMAX ? !(most < INFINITY) : isnan(most); // (the softmax of infinity is NaN)
  if (lost) best = most_of(l);
  if (SOFTMAX && (BIAS || !normalise)) {
    top = warp_most(best);
    if (top > -INFINITY) {
#pragma unroll
      for (int j = 0; j < J; ++j) sum += expf(l[j] - top);
      sum = warp_sum(sum);
    }
  }
  float mine;
  int expert, found;
  if constexpr (!BIAS) {
    found = candidates(l, best, k, list, [](float b) { return b; }, mine, expert);
    if (found > 32) {
      unsigned key[J];
#pragma unroll
      for (int j = 0; j < J; ++j) key[j] = ordered(l[j]);
      expert = greatest(key, k);
      mine = expert >= 0 ? to_float(own[MS_AT(expert, E)]) : -INFINITY;
    }
  } else {
    float key[J];
    load_logits(bias, E, J % 4 == 0 && E % 4 == 0 && (reinterpret_cast<uintptr_t>(bias) & 15) == 0, key);
    const float share = SOFTMAX ? __fdividef(1.0f, sum) : 0.0f;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const float s = SOFTMAX ? rough_exponential(l[j] - top) * share : rough_logistic(l[j]);
      key[j] = l[j] > -INFINITY ? s + key[j] : -INFINITY;
    }
    found = candidates(key, most_of(key), k, list, [](float b) { return b - 2.0f * apart(b, b); }, mine, expert);
    const float next = __shfl_down_sync(FULL, mine, 1);
    const bool near = lane < k && lane + 1 < found && !(mine - next > apart(mine, next));
    mine = expert >= 0 ? to_float(own[MS_AT(expert, E)]) : -INFINITY;
    if (SOFTMAX && lost) {                                      // (no key is a number)
      expert = choose_lost(l, bias, E, k);
      mine = expert >= 0 ? to_float(own[MS_AT(expert, E)]) : -INFINITY;
    } else if (found > 32 || __any_sync(FULL, near)) {
      const double wide_sum = SOFTMAX ? softmax_sum64(l, top) : 1.0;
      expert = found > 32 ? choose64<J, SCORE>(l, bias, E, k, top, wide_sum)
                          : order64<SCORE>(mine, expert >= 0 ? bias[MS_AT(expert, E)] : 0.0f, top, wide_sum, expert, found, list);
      mine = expert >= 0 ? to_float(own[MS_AT(expert, E)]) : -INFINITY;
    }
  }
  const bool there = lane < k && expert >= 0;
  if (!there) mine = -INFINITY;
  const float w = normalise ? normalised<SOFTMAX>(mine, there) : SOFTMAX ? quotient(expf(mine - top), sum) : logistic(mine);
  if (lane < k) {
    experts[row * k + lane] = there ? expert : -1;
    weights[row * k + lane] = lost ? NAN : there ? w * factor : 0.0f;
  }
}

// Gradients of the logits, from a = factor * dw:
//   softmax             p (a [chosen] - sum a p)      over all experts
//   softmax, normalised q (a - sum a q)               over the chosen, 0 for the others
//   logistic            a s (1 - s);  normalised  q (a - sum a q) (1 - s)
template <typename T, int J, int SCORE>
__global__ void __launch_bounds__(32 * CHOOSE_WARPS) choose_backward_kernel(int rows, int E, int k, int normalise, int wide, float factor,
                                                                            const float* __restrict__ dweights,
                                                                            const T* __restrict__ logits,
                                                                            const int32_t* __restrict__ experts, T* dlogits) {
  constexpr bool SOFTMAX = SCORE == MOESCHED_SCORE_SOFTMAX;
  constexpr int COUNT = Vec<T>::COUNT;
  const int lane = threadIdx.x & 31;
  const long long row = (long long)blockIdx.x * CHOOSE_WARPS + (threadIdx.x >> 5);
  if (row >= rows) return;
  const T* own = logits + row * E;
  T* out = dlogits + row * E;
  int expert = lane < k ? experts[row * k + lane] : -1;
  float a = lane < k ? dweights[row * k + lane] * factor : 0.0f;
  const bool all = SOFTMAX && !normalise;
  if (!all) {                                                    // zeros, while the choices are on their way
    if (wide)
      for (int e = lane * COUNT; e < E; e += 32 * COUNT) *reinterpret_cast<uint4*>(out + e) = make_uint4(0u, 0u, 0u, 0u);
    else
      for (int e = lane; e < E; e += 32) put(out + e, 0.0f);
  }
  if ((unsigned)expert >= (unsigned)E) expert = -1;
  const bool there = expert >= 0;
  const float mine = there ? to_float(own[MS_AT(expert, E)]) : -INFINITY;
  a = there ? a : 0.0f;
  float d;
  if (all) {
    float l[J], top, sum;
    load_logits(own, E, wide != 0, l);
    softmax_of(l, top, sum);
    const float share = 1.0f / sum, p = there ? expf(mine - top) * share : 0.0f, dot = warp_sum(a * p);
    d = p * (a - dot);
#pragma unroll
    for (int j = 0; j < J; ++j) l[j] = l[j] == -INFINITY ? 0.0f : expf(l[j] - top) * share * -dot;
    if (J % COUNT == 0 && wide) {
#pragma unroll
      for (int j = 0; j < J; j += COUNT) {
        float f[COUNT];
#pragma unroll
        for (int q = 0; q < COUNT; ++q) f[q] = l[(j + q) % J];
        if (lane * J + j < E) *reinterpret_cast<uint4*>(out + lane * J + j) = Vec<T>::pack(f);
      }
    } else {
#pragma unroll
      for (int j = 0; j < J; ++j)
        if (lane * J + j < E) put(out + lane * J + j, l[j]);
    }
  } else if (normalise) {
    const float q = normalised<SOFTMAX>(mine, there), dot = warp_sum(there ? a * q : 0.0f);
    d = q * (a - dot);
    if (!SOFTMAX) d *= logistic(-mine);
  } else {
    d = a * logistic_slope(mine);
  }
  __syncwarp();                                                  // the chosen after all of them
  if (there) put(out + MS_AT(expert, E), d);
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

// Rows of logits start and end on 16 bytes
template <typename T>
static bool wide_rows(int E, const void* p, const void* q) {
  return E % Vec<T>::COUNT == 0 && (reinterpret_cast<uintptr_t>(p) | reinterpret_cast<uintptr_t>(q)) % 16 == 0;
}

cudaError_t run_choose(int rows, int E, int k, int dtype, int score, int normalise, float factor, const void* logits, const float* bias,
                       int32_t* experts, float* weights, cudaStream_t stream) {
  return with_type(dtype, [&](auto type) {
    using T = decltype(type);
    return with_experts(E, [&](auto count) {
      constexpr int J = decltype(count)::value;
      constexpr int SOFTMAX = MOESCHED_SCORE_SOFTMAX, SIGMOID = MOESCHED_SCORE_SIGMOID;
      const auto kern = score == SOFTMAX ? (bias != nullptr ? choose_kernel<T, J, SOFTMAX, true> : choose_kernel<T, J, SOFTMAX, false>)
                                         : (bias != nullptr ? choose_kernel<T, J, SIGMOID, true> : choose_kernel<T, J, SIGMOID, false>);
      return launch(kern, dim3((rows + CHOOSE_WARPS - 1) / CHOOSE_WARPS), dim3(32 * CHOOSE_WARPS), 0, false, stream, rows, E, k, normalise,
                    (int)wide_rows<T>(E, logits, nullptr), factor, static_cast<const T*>(logits), bias, experts, weights);
    });
  });
}

cudaError_t run_choose_backward(int rows, int E, int k, int dtype, int score, int normalise, float factor, const float* dweights,
                                const void* logits, const int32_t* experts, void* dlogits, cudaStream_t stream) {
  return with_type(dtype, [&](auto type) {
    using T = decltype(type);
    return with_experts(E, [&](auto count) {
      constexpr int J = decltype(count)::value;
      const auto kern = score == MOESCHED_SCORE_SOFTMAX ? choose_backward_kernel<T, J, MOESCHED_SCORE_SOFTMAX>
                                                        : choose_backward_kernel<T, J, MOESCHED_SCORE_SIGMOID>;
      return launch(kern, dim3((rows + CHOOSE_WARPS - 1) / CHOOSE_WARPS), dim3(32 * CHOOSE_WARPS), 0, false, stream, rows, E, k, normalise,
                    (int)wide_rows<T>(E, logits, dlogits), factor, dweights, static_cast<const T*>(logits), experts, static_cast<T*>(dlogits));
    });
  });
}

}  // namespace moesched
