// Router's choices to demand: a stable counting sort of every source rank's choices by expert.
//
// For source i of matrix b, e[s] = expert of choice s (or none):
//   counts[x] = #{s : e[s] = x},   demand[j] = sum of counts over the experts of rank j,
//   slot[s]   = #{s' : e[s'] < e[s]} + #{s' < s : e[s'] = e[s]}      (its place in the send buffer)
// One CTA owns one source. Its warps own consecutive stretches of the choices and a histogram each (shared memory); a
// scan over experts, and for each expert over the warps, turns the histograms into first slots; then every warp walks its stretch
// again, 32 choices at a time, and ranks equal choices with a vote, so that the order is that of the choices and nothing depends
// on the order of atomics. Bound by memory: 4 bytes in (the second walk finds them in L2) and 4 out for each choice.
#include "common.cuh"

namespace moesched {

constexpr int ROUTE_AHEAD = 4;   // loads in flight per lane

template <int WARPS>
__global__ void __launch_bounds__(32 * WARPS) route_kernel(int N, int S, int E, const int32_t* __restrict__ experts,
                                                           int32_t* __restrict__ demand, int32_t* __restrict__ counts,
                                                           int32_t* __restrict__ slot, int32_t* __restrict__ status) {
  extern __shared__ int shared[];
  int* warp_sum = shared;                    // [WARPS]
  int* hist = shared + WARPS;                // [WARPS][E]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const size_t src = blockIdx.x;             // b * N + i
  const int32_t* in = experts + src * S;
  int32_t* out = slot + src * S;
  int* mine = hist + warp * E;
  for (int x = threadIdx.x; x < WARPS * E; x += 32 * WARPS) hist[x] = 0;
  __syncthreads();
  // stretches of whole groups of 32, so that a warp's accesses stay together
  const int per = ((S + WARPS - 1) / WARPS + 31) / 32 * 32;
  const int begin = (int)min((long long)S, (long long)warp * per), end = (int)min((long long)S, (long long)begin + per);
  bool bad = false;
  for (int s0 = begin; s0 < end; s0 += 32 * ROUTE_AHEAD) {
    int e[ROUTE_AHEAD];
#pragma unroll
    for (int q = 0; q < ROUTE_AHEAD; ++q) {
      const int s = s0 + 32 * q + lane;
      e[q] = s < end ? in[s] : -1;
    }
#pragma unroll
    for (int q = 0; q < ROUTE_AHEAD; ++q) {
      if ((unsigned)e[q] < (unsigned)E) atomicAdd(&mine[MS_AT(e[q], E)], 1);
      else bad |= e[q] != -1;
    }
  }
  bad = __syncthreads_or(bad);
  // totals, first slots: thread t has the experts t, t + threads, ... in rounds, with the sum of the rounds before
  int base = 0;
  for (int x0 = 0; x0 < E; x0 += 32 * WARPS) {
    const int x = x0 + threadIdx.x;
    int total = 0;
    if (x < E) {
#pragma unroll 8
      for (int w = 0; w < WARPS; ++w) total += hist[w * E + x];
      counts[src * E + x] = total;
    }
    int incl = total;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(FULL, incl, o);
      if (lane >= o) incl += v;
    }
    if (lane == 31) warp_sum[warp] = incl;
    __syncthreads();
    int before = base, all = base;
#pragma unroll 8
    for (int w = 0; w < WARPS; ++w) {
      const int v = warp_sum[w];
      before += w < warp ? v : 0;
      all += v;
    }
    int first = before + incl - total;
    if (x < E) {
#pragma unroll 8
      for (int w = 0; w < WARPS; ++w) {
        const int v = hist[w * E + x];
        hist[w * E + x] = first;
        first += v;
      }
    }
    base = all;
    __syncthreads();
  }
  // hist[0][x] is the first slot of expert x: differences over the experts of a rank are the demand
  const int P = E / N;
  for (int j = threadIdx.x; j < N; j += 32 * WARPS)
    demand[src * N + j] = (j + 1 < N ? hist[(j + 1) * P] : base) - hist[j * P];
  if (threadIdx.x == 0) status[src] = bad ? MOESCHED_ST_BAD_INPUT : MOESCHED_ST_OK;
  __syncthreads();   // (warp 0 moves its first slots on)
  for (int s0 = begin; s0 < end; s0 += 32 * ROUTE_AHEAD) {
    int e[ROUTE_AHEAD];
#pragma unroll
    for (int q = 0; q < ROUTE_AHEAD; ++q) {
      const int s = s0 + 32 * q + lane;
      e[q] = s < end ? in[s] : -1;
    }
#pragma unroll
    for (int q = 0; q < ROUTE_AHEAD; ++q) {
      const int s = s0 + 32 * q + lane;
      const bool sent = (unsigned)e[q] < (unsigned)E;
      const unsigned peers = __match_any_sync(FULL, sent ? e[q] : -1);
      const int rank = __popc(peers & ((1u << lane) - 1));
      const int first = sent ? mine[MS_AT(e[q], E)] : 0;
      __syncwarp();
      if (sent && rank == 0) mine[MS_AT(e[q], E)] = first + __popc(peers);
      __syncwarp();
      if (s < end) out[s] = sent ? first + rank : -1;
    }
  }
}

cudaError_t run_route(int B, int N, int S, int E, const int32_t* experts, int32_t* demand, int32_t* counts, int32_t* slot,
                      int32_t* status, cudaStream_t stream) {
  constexpr int WARPS = 32;
  const auto kern = route_kernel<WARPS>;
  const size_t smem = (size_t)WARPS * (E + 1) * sizeof(int);
  if (cudaError_t e = permit_shared_memory(kern, smem); e != cudaSuccess) return e;
  kern<<<(unsigned)(B * N), 32 * WARPS, smem, stream>>>(N, S, E, experts, demand, counts, slot, status);
  return cudaGetLastError();
}

}  // namespace moesched
