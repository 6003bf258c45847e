// Products of a few rows with the weights of their experts: y = x W^T, or act(x Wg^T) * (x Wu^T), W in 16 bits, or in 4 bits
// with a scale for every group of weights along k, w = (q - 8) * scale.
//
// With a handful of rows the weights' bytes are all that counts. A warp streams 16 rows of the weights of one expert
// from global memory straight into the operand registers of the matrix instruction (16 x 8 x 16: the weights are its
// 16 rows, up to eight tokens its columns), so that a weight is handled once for all eight tokens. Which k a lane holds is free as
// long as both operands agree on it: a lane's 16-byte load is eight (4 bits: 32) neighbouring k, and x is loaded to
// match. In 4 bits an instruction never mixes the groups of scales: the sum over one group is made in 32 bits of (q - 8) x,
// which 16-bit operands hold exactly, and scaled when it is added up. The warps of a CTA share the k of the same outputs (`split`
// of them) and add up in shared memory in a fixed order.
#include "expert.cuh"

namespace moesched {

constexpr int FEW_WARPS = 8;
constexpr int FEW_ROWS = 8;      // tokens per pass over the weights

struct FewArgs {
  int R, K, N, E, groups, split;
  const void *x, *w[2], *scale[2];
  const int32_t* offsets;
  void *y, *sum[2];              // sum: the two products themselves, where they are wanted (16 bits)
  int32_t* status;
};

template <typename T>
__device__ __forceinline__ void mma16816(float (&c)[4], const unsigned (&a)[4], unsigned b0, unsigned b1) {
  if constexpr (sizeof(T) == 2 && std::is_same_v<T, __half>)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Four pairs (q0, q4), (q1, q5), (q2, q6), (q3, q7) of a word of eight 4-bit numbers, minus 8: a number under the
// leading bit of 2^7 (bfloat16) or 2^10 (half) is that power plus itself, and the difference of two such is exact.
template <typename T>
__device__ __forceinline__ void unpack4(unsigned w, unsigned (&v)[4]) {
  constexpr bool HALF = std::is_same_v<T, __half>;
  constexpr unsigned LEAD = HALF ? 0x64006400u : 0x43004300u, EIGHT = HALF ? 0x64086408u : 0x43084308u;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    unsigned u = ((w >> (4 * q)) & 0x000f000fu) | LEAD;
    if constexpr (HALF) {
      const __half2 d = __hsub2(*reinterpret_cast<const __half2*>(&u), *reinterpret_cast<const __half2*>(&EIGHT));
      v[q] = *reinterpret_cast<const unsigned*>(&d);
    } else {
      const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&u), *reinterpret_cast<const __nv_bfloat162*>(&EIGHT));
      v[q] = *reinterpret_cast<const unsigned*>(&d);
    }
  }
}

template <int WORDS>
__device__ __forceinline__ void load_stream(const void* p, unsigned (&v)[WORDS]) {
  if constexpr (WORDS == 4)
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "l"(p));
  else if constexpr (WORDS == 2)
    asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(v[0]), "=r"(v[1]) : "l"(p));
  else
    asm volatile("ld.global.nc.u32 %0, [%1];" : "=r"(v[0]) : "l"(p));
}

// GROUP: weights per scale, 0 for weights in 16 bits
template <typename T, int GROUP, bool GATED, int ACT>
__global__ void __launch_bounds__(32 * FEW_WARPS) few_kernel(const FewArgs a) {
  constexpr bool Q4 = GROUP != 0;
  constexpr int MATS = GATED ? 2 : 1;
  constexpr int BLOCK = Q4 ? 128 : 64;                 // k per step of a warp
  constexpr int PIECES = Q4 ? BLOCK / GROUP : BLOCK / 32;   // stretches of k that a load instruction covers with four lanes
  constexpr int EACH = BLOCK / 4 / PIECES;             // neighbouring k of a lane in a stretch
  constexpr int WORDS = Q4 ? EACH / 8 : EACH / 2;      // 32-bit words of weights of a lane in a stretch
  __shared__ int rows[FEW_ROWS];
  __shared__ int row_count;
  __shared__ float sums[FEW_WARPS][MATS][FEW_ROWS][16];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int e = blockIdx.y, R = a.R, K = a.K, N = a.N;
  const int split = a.split, part = warp % split, tile = warp / split;
  const int n0 = (blockIdx.x * (FEW_WARPS / split) + tile) * 16;
  const int gr = lane >> 2, t = lane & 3;
  const T* x = static_cast<const T*>(a.x);

  if (blockIdx.x == 0 && e == 0) {                     // one CTA looks at all offsets
    bool bad = false;
    for (int g = threadIdx.x; g <= a.groups; g += 32 * FEW_WARPS) {
      const int v = a.offsets[g];
      bad |= v < 0 || v > R || (g > 0 && a.offsets[g - 1] > v);
    }
    bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) *a.status = bad ? MOESCHED_ST_BAD_INPUT : MOESCHED_ST_OK;
  }

  const size_t row_bytes = Q4 ? (size_t)K / 2 : (size_t)K * 2;
  const char* wrow[MATS][2];
  const T* srow[MATS][2];
#pragma unroll
  for (int m = 0; m < MATS; ++m)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const size_t n = (size_t)e * N + min(n0 + gr + 8 * h, N - 1);
      wrow[m][h] = static_cast<const char*>(a.w[m]) + n * row_bytes;
      if constexpr (Q4) srow[m][h] = static_cast<const T*>(a.scale[m]) + n * (K / (Q4 ? GROUP : 1));
    }

  for (int skip = 0; skip < R; skip += FEW_ROWS) {     // (offsets out of order may name more rows than there are)
    // the next rows of the expert, over its groups
    __syncthreads();
    if (warp == 0) {
      if (lane < FEW_ROWS) rows[lane] = -1;
      __syncwarp();
      int seen = 0;
      for (int g0 = e; g0 < a.groups && seen < skip + FEW_ROWS; g0 += 32 * a.E) {
        const long long g = g0 + (long long)lane * a.E;
        const int2 span = g < a.groups ? rows_of_group(a.offsets, (int)g, R) : make_int2(0, 0);
        const int len = span.y - span.x;
        int incl = len;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int v = __shfl_up_sync(FULL, incl, o);
          if (lane >= o) incl += v;
        }
        // (well-formed offsets add up to at most R; others may wrap, and then some rows are passed over)
        const int first = seen + incl - len;
        for (int q = 0; q < FEW_ROWS; ++q) {
          const int at = skip + q - first;
          if (at >= 0 && at < len) rows[q] = span.x + at;
        }
        seen += __shfl_sync(FULL, incl, 31);
      }
      __syncwarp();
      if (lane == 0) row_count = max(0, min(FEW_ROWS, seen - skip));
    }
    __syncthreads();
    const int count = row_count;
    if (count == 0) break;
    const int my_row = rows[gr];
    const T* xrow = x + (size_t)max(my_row, 0) * K;

    float acc[MATS][4];
#pragma unroll
    for (int m = 0; m < MATS; ++m)
#pragma unroll
      for (int q = 0; q < 4; ++q) acc[m][q] = 0.0f;

    struct Held {
      unsigned w[MATS][2][PIECES][WORDS];
      unsigned x[PIECES][EACH / 2];
      T s[MATS][2][PIECES];
    };
    auto load = [&](int k0, Held& h) {
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        const int k = k0 + p * 4 * EACH + t * EACH;
        const bool in = k < K;
#pragma unroll
        for (int q = 0; q < EACH / 8; ++q) {
          uint4 v = make_uint4(0, 0, 0, 0);
          if (in && my_row >= 0) v = *reinterpret_cast<const uint4*>(xrow + k + 8 * q);
          h.x[p][4 * q] = v.x, h.x[p][4 * q + 1] = v.y, h.x[p][4 * q + 2] = v.z, h.x[p][4 * q + 3] = v.w;
        }
#pragma unroll
        for (int m = 0; m < MATS; ++m)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
#pragma unroll
            for (int q = 0; q < WORDS; ++q) h.w[m][r][p][q] = 0;
            if (in) load_stream(wrow[m][r] + (Q4 ? (size_t)k / 2 : (size_t)k * 2), h.w[m][r][p]);
            if constexpr (Q4) {
              if (in) h.s[m][r][p] = srow[m][r][k / (Q4 ? GROUP : 1)];
              else put(&h.s[m][r][p], 0.0f);
            }
          }
      }
    };
    auto multiply = [&](const Held& h) {
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        float sum[MATS][4];
#pragma unroll
        for (int m = 0; m < MATS; ++m)
#pragma unroll
          for (int q = 0; q < 4; ++q) sum[m][q] = Q4 ? 0.0f : acc[m][q];
#pragma unroll
        for (int q = 0; q < EACH / 8; ++q) {
          unsigned xv[4];
          if constexpr (Q4) {      // x in the order of unpack4's pairs
            xv[0] = __byte_perm(h.x[p][4 * q], h.x[p][4 * q + 2], 0x5410);
            xv[1] = __byte_perm(h.x[p][4 * q], h.x[p][4 * q + 2], 0x7632);
            xv[2] = __byte_perm(h.x[p][4 * q + 1], h.x[p][4 * q + 3], 0x5410);
            xv[3] = __byte_perm(h.x[p][4 * q + 1], h.x[p][4 * q + 3], 0x7632);
          } else {
#pragma unroll
            for (int c = 0; c < 4; ++c) xv[c] = h.x[p][4 * q + c];
          }
#pragma unroll
          for (int m = 0; m < MATS; ++m) {
            unsigned lo[4], hi[4];
            if constexpr (Q4) {
              unpack4<T>(h.w[m][0][p][q], lo);
              unpack4<T>(h.w[m][1][p][q], hi);
            } else {
#pragma unroll
              for (int c = 0; c < 4; ++c) lo[c] = h.w[m][0][p][4 * q + c], hi[c] = h.w[m][1][p][4 * q + c];
            }
            const unsigned f0[4] = {lo[0], hi[0], lo[1], hi[1]}, f1[4] = {lo[2], hi[2], lo[3], hi[3]};
            mma16816<T>(sum[m], f0, xv[0], xv[1]);
            mma16816<T>(sum[m], f1, xv[2], xv[3]);
          }
        }
#pragma unroll
        for (int m = 0; m < MATS; ++m) {
          const float s0 = Q4 ? to_float(h.s[m][0][p]) : 1.0f, s1 = Q4 ? to_float(h.s[m][1][p]) : 1.0f;
#pragma unroll
          for (int q = 0; q < 4; ++q) acc[m][q] = Q4 ? fmaf(q < 2 ? s0 : s1, sum[m][q], acc[m][q]) : sum[m][q];
        }
      }
    };
    if (n0 < N) {
      Held h[2];
      const int step = BLOCK * split;
      int k = part * BLOCK;
      if (k < K) load(k, h[0]);
      while (k < K) {
        if (k + step < K) load(k + step, h[1]);
        multiply(h[0]);
        k += step;
        if (k >= K) break;
        if (k + step < K) load(k + step, h[0]);
        multiply(h[1]);
        k += step;
      }
    }
    // lane (gr, t) has outputs gr, gr + 8 of the tokens 2t, 2t + 1
#pragma unroll
    for (int m = 0; m < MATS; ++m)
#pragma unroll
      for (int q = 0; q < 4; ++q) sums[warp][m][2 * t + (q & 1)][gr + 8 * (q >> 1)] = acc[m][q];
    __syncthreads();
    const int tiles = FEW_WARPS / split;
    for (int q = threadIdx.x; q < tiles * FEW_ROWS * 16; q += 32 * FEW_WARPS) {
      const int c = q % 16, tl = q / 16 % tiles, r = q / (16 * tiles);
      const int n = (blockIdx.x * tiles + tl) * 16 + c;
      if (r >= count || n >= N) continue;
      float v[MATS];
#pragma unroll
      for (int m = 0; m < MATS; ++m) {
        v[m] = 0.0f;
        for (int s = 0; s < split; ++s) v[m] += sums[tl * split + s][m][r][c];
      }
      const size_t to = (size_t)rows[r] * N + n;
      if constexpr (GATED) {
        if (a.sum[0] != nullptr) {
          put(static_cast<T*>(a.sum[0]) + to, v[0]);
          put(static_cast<T*>(a.sum[1]) + to, v[1]);
        }
        put(static_cast<T*>(a.y) + to, activation<ACT>(v[0]) * v[1]);
      } else {
        put(static_cast<T*>(a.y) + to, v[0]);
      }
    }
  }
}

template <typename T, int GROUP>
static cudaError_t launch_few(const FewArgs& a, bool gated, int act, cudaStream_t stream) {
  const int tiles = FEW_WARPS / a.split;
  const dim3 grid((unsigned)((a.N + 16 * tiles - 1) / (16 * tiles)), (unsigned)a.E);
  if (!gated) few_kernel<T, GROUP, false, MOESCHED_ACT_SILU><<<grid, 32 * FEW_WARPS, 0, stream>>>(a);
  else if (act == MOESCHED_ACT_SILU) few_kernel<T, GROUP, true, MOESCHED_ACT_SILU><<<grid, 32 * FEW_WARPS, 0, stream>>>(a);
  else few_kernel<T, GROUP, true, MOESCHED_ACT_GELU><<<grid, 32 * FEW_WARPS, 0, stream>>>(a);
  return cudaGetLastError();
}

cudaError_t run_few(int R, int K, int N, int E, int groups, int group, int dtype, int act, const void* x, const void* w,
                    const void* scale, const void* w_up, const void* scale_up, const int32_t* offsets, void* y, void* sum,
                    void* sum_up, int32_t* status, cudaStream_t stream) {
  FewArgs a{R, K, N, E, groups, 1, x, {w, w_up}, {scale, scale_up}, offsets, y, {sum, sum_up}, status};
  // as few warps share the k of an output as still give every SM two CTAs
  const long long tiles = (long long)(E < R ? E : R) * ((N + 15) / 16);
  while (a.split < FEW_WARPS && tiles * a.split < 2LL * FEW_WARPS * sm_count()) a.split *= 2;
  const bool gated = w_up != nullptr;
  if (dtype == MOESCHED_BF16) {
    if (group == 0) return launch_few<__nv_bfloat16, 0>(a, gated, act, stream);
    if (group == 32) return launch_few<__nv_bfloat16, 32>(a, gated, act, stream);
    if (group == 64) return launch_few<__nv_bfloat16, 64>(a, gated, act, stream);
    return launch_few<__nv_bfloat16, 128>(a, gated, act, stream);
  }
  if (group == 0) return launch_few<__half, 0>(a, gated, act, stream);
  if (group == 32) return launch_few<__half, 32>(a, gated, act, stream);
  if (group == 64) return launch_few<__half, 64>(a, gated, act, stream);
  return launch_few<__half, 128>(a, gated, act, stream);
}

}  // namespace moesched
