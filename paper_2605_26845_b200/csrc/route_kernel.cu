// Router's choices to demand: a stable counting sort of every source rank's choices by expert.
//
// For source i of matrix b, e[s] = expert of choice s (or none):
//   counts[x] = #{s : e[s] = x},   demand[j] = sum of counts over the experts of rank j,
//   slot[s]   = #{s' : e[s'] < e[s]} + #{s' < s : e[s'] = e[s]}      (its place in the send buffer)
// One CTA owns one source, or a cluster of them where there are few. Its warps own consecutive stretches of the choices and a
// table each (shared memory) with a counter and 32 bits for every expert. A scan over experts, and for each expert over
// the warps (and CTAs), turns the counters into first slots. Then every warp walks its stretch again, 32 choices at a time: each
// lane sets its bit at its expert, reads the bits of the others there and the slot, and the lowest moves the slot on. So the order is
// that of the choices, and nothing depends on the order of atomics. 4 bytes in, twice, and 4 out for each choice, and 16 or so
// accesses to shared memory for 32 choices, which bound it: 64 ranks x 16 layers x 131072 choices
// of 256 experts take 410 us, 637 of 820 thousand cycles in shared memory (votes on equal values in place of the bits, match: twice as
// long; votes on each bit of the number 1.9 times). The bytes alone, read once, would take 167 us.
#include "common.cuh"

namespace moesched {

constexpr int ROUTE_AHEAD = 4;   // loads in flight per lane (8: 5 % more time)

// table: x bits of the lanes that hold the expert now, y counter, then next slot
template <int WARPS>
__global__ void __launch_bounds__(32 * WARPS) route_kernel(int N, int S, int E, int CS, const int32_t* __restrict__ experts,
                                                           int32_t* __restrict__ demand, int32_t* __restrict__ counts,
                                                           int32_t* __restrict__ slot, int32_t* __restrict__ status) {
  extern __shared__ __align__(8) int shared[];
  int* warp_sum = shared;                                   // [WARPS]
  int* own = shared + WARPS;                                // [E + 1] this CTA's counts, and whether it saw a bad choice
  uint2* table = reinterpret_cast<uint2*>(shared + WARPS + (E + 2) / 2 * 2);   // [WARPS][E]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int part = blockIdx.x % CS;
  const size_t src = blockIdx.x / CS;                       // b * N + i
  const int32_t* in = experts + src * S;
  int32_t* out = slot + src * S;
  uint2* mine = table + warp * E;
  for (int x = threadIdx.x; x < WARPS * E; x += 32 * WARPS) table[x] = make_uint2(0u, 0u);
  __syncthreads();
  // stretches of whole groups of 32, so that a warp's accesses stay together
  const long long all_warps = (long long)WARPS * CS, at = (long long)part * WARPS + warp;
  const long long per = ((S + all_warps - 1) / all_warps + 31) / 32 * 32;
  const int begin = (int)min((long long)S, at * per), end = (int)min((long long)S, (at + 1) * per);
  const int rounds = (end - begin + 32 * ROUTE_AHEAD - 1) / (32 * ROUTE_AHEAD);
  bool bad = false;
  const auto load = [&](int round, int (&e)[ROUTE_AHEAD]) {
#pragma unroll
    for (int q = 0; q < ROUTE_AHEAD; ++q) {
      const int o = 32 * (round * ROUTE_AHEAD + q) + lane;
      e[q] = o < end - begin ? in[begin + o] : -1;
    }
  };
  for (int r = 0; r < rounds; ++r) {
    int e[ROUTE_AHEAD];
    load(r, e);
#pragma unroll
    for (int q = 0; q < ROUTE_AHEAD; ++q) {
      if ((unsigned)e[q] < (unsigned)E) atomicAdd(&mine[MS_AT(e[q], E)].y, 1u);
      else bad |= e[q] != -1;
    }
  }
  bad = __syncthreads_or(bad);
  if (CS > 1) {
    for (int x = threadIdx.x; x < E; x += 32 * WARPS) {
      int total = 0;
#pragma unroll 8
      for (int w = 0; w < WARPS; ++w) total += (int)table[w * E + x].y;
      own[x] = total;
    }
    if (threadIdx.x == 0) own[E] = bad;
    __syncwarp();                                           // (a cluster's barrier is for whole warps)
    cluster_sync_all();
  }
  // totals, first slots: thread t has the experts t, t + threads, ... in rounds, with the sum of the rounds before
  int base = 0;
  for (int x0 = 0; x0 < E; x0 += 32 * WARPS) {
    const int x = x0 + threadIdx.x;
    int total = 0, skipped = 0;                             // skipped: the choices of the CTAs before this one
    if (x < E) {
      if (CS > 1) {
        for (int c = 0; c < CS; ++c) {
          const int v = *map_to_cta(own + x, c);
          total += v;
          skipped += c < part ? v : 0;
        }
      } else {
#pragma unroll 8
        for (int w = 0; w < WARPS; ++w) total += (int)table[w * E + x].y;
      }
      if (part == 0) counts[src * E + x] = total;
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
    unsigned first = (unsigned)(before + incl - total + skipped);
    if (x < E) {
#pragma unroll 8
      for (int w = 0; w < WARPS; ++w) {
        const unsigned v = table[w * E + x].y;
        table[w * E + x].y = first;
        first += v;
      }
    }
    base = all;
    __syncthreads();
  }
  if (part == 0) {
    // table[0][x] is the first slot of expert x: differences over the experts of a rank are the demand
    const int P = E / N;
    for (int j = threadIdx.x; j < N; j += 32 * WARPS)
      demand[src * N + j] = (j + 1 < N ? (int)table[(j + 1) * P].y : base) - (int)table[j * P].y;
    if (threadIdx.x == 0) {
      for (int c = 1; c < CS; ++c) bad |= *map_to_cta(own + E, c) != 0;
      status[src] = bad ? MOESCHED_ST_BAD_INPUT : MOESCHED_ST_OK;
    }
  }
  __syncwarp();
  if (CS > 1) cluster_sync_all();                           // (nobody leaves while others read)
  else __syncthreads();                                     // (warp 0 moves its first slots on)
  const unsigned below = (1u << lane) - 1;
  for (int r = 0; r < rounds; ++r) {
    int e[ROUTE_AHEAD];
    load(r, e);
#pragma unroll
    for (int q = 0; q < ROUTE_AHEAD; ++q) {
      const int o = 32 * (r * ROUTE_AHEAD + q) + lane;
      const bool sent = (unsigned)e[q] < (unsigned)E;
      uint2* to = mine + MS_AT(sent ? e[q] : 0, E);
      if (sent) atomicOr(&to->x, 1u << lane);
      __syncwarp();
      const unsigned long long word = *reinterpret_cast<volatile unsigned long long*>(to);
      const unsigned peers = (unsigned)word, first = (unsigned)(word >> 32);
      const int rank = __popc(peers & below);
      __syncwarp();
      if (sent && rank == 0) *to = make_uint2(0u, first + __popc(peers));
      __syncwarp();
      if (o < end - begin) out[begin + o] = sent ? (int)first + rank : -1;
    }
  }
}

template <int WARPS>
static cudaError_t launch_route(int B, int N, int S, int E, const int32_t* experts, int32_t* demand, int32_t* counts,
                                int32_t* slot, int32_t* status, cudaStream_t stream) {
  const auto kern = route_kernel<WARPS>;
  const size_t smem = ((size_t)WARPS + (E + 2) / 2 * 2) * sizeof(int) + (size_t)WARPS * E * sizeof(uint2);
  if (cudaError_t e = permit_shared_memory(kern, smem); e != cudaSuccess) return e;
  // few sources: several CTAs for each, with a few thousand choices at least
  int CS = 1;
  while (CS < 8 && (long long)B * N * CS * 2 <= sm_count() && S / CS >= 8192) CS *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((long long)B * N * CS));
  cfg.blockDim = dim3(32 * WARPS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  if (CS > 1) {
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = CS;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
  }
  return cudaLaunchKernelEx(&cfg, kern, N, S, E, CS, experts, demand, counts, slot, status);
}

cudaError_t run_route(int B, int N, int S, int E, const int32_t* experts, int32_t* demand, int32_t* counts, int32_t* slot,
                      int32_t* status, cudaStream_t stream) {
  // the tables of 32 warps for up to 256 experts let an SM hold two CTAs; those of 16 warps for 1024 fit one
  return E <= 256 ? launch_route<32>(B, N, S, E, experts, demand, counts, slot, status, stream)
                  : launch_route<16>(B, N, S, E, experts, demand, counts, slot, status, stream);
}

}  // namespace moesched
