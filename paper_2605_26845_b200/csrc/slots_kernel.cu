// Where the tokens of a schedule go: its replay against the demand, with the place of every transfer.
//
// With j = pi_k(i), used = tokens of the pair (i, j) that matchings before k have carried:
//   start  = min(D_ij, used),  length = min(D_ij - start, dur_k),  row = tokens that j has received before matching k,
//   offsets[j][k P + e] = row + (tokens of the transfer that are for experts of j below e); a pair's tokens lie by expert.
// A pair's transfers depend on one another only through `used`, a receiver's rows only through a running sum. So a CTA takes 32
// matchings at a time: a warp per source with a lane per matching (equal destinations among the 32 are summed by votes), then a warp
// per receiver with a lane per matching and a prefix sum over the lanes, then coalesced stores by matching. The pairs'
// `used` and demand are in shared memory.
#include "common.cuh"

namespace moesched {

constexpr int SLOT_CHUNK = 32;         // matchings per step: one per lane
constexpr int SLOT_FUSED_N = 128;      // up to here the pairs of a whole matrix fit one CTA's shared memory
constexpr int SLOT_BLOCK = 64;         // sources per CTA above

struct SlotArgs {
  int N, K, P, CS;                     // CS: CTAs of a cluster, each with a stretch of the matchings
  const int32_t* demand;
  const uint8_t* perm;
  const int32_t* dur;
  const int32_t* count;
  const int32_t* counts;               // [B][N][N * P] or NULL
  int32_t *start, *length, *row, *rows, *offsets, *status;
};

// strides in shared memory that put the 32 lanes' accesses to one column into different banks
__host__ __device__ inline int slot_int_stride(int N) { return N | 1; }
__host__ __device__ inline int slot_byte_stride(int N) { return 4 * (((N + 3) / 4) | 1); }

struct SlotSmem {
  size_t pairs, received, start, len, begins, perm, source, dur, bad, bytes;
};
// `sources` in this CTA (with their pairs if it walks them), and `receivers` (all of them, or none)
__host__ __device__ inline SlotSmem slot_smem(int N, int sources, bool pairs, int receivers) {
  SlotSmem m;
  size_t at = 0;
  m.pairs = at, at += pairs ? align16((size_t)sources * N * sizeof(int2)) : 0;
  m.received = at, at += align16((size_t)receivers * sizeof(long long));
  m.start = at, at += align16((size_t)SLOT_CHUNK * slot_int_stride(sources) * 4);
  m.len = at, at += align16((size_t)SLOT_CHUNK * slot_int_stride(sources) * 4);
  m.begins = at, at += align16((size_t)SLOT_CHUNK * slot_int_stride(receivers) * 4);
  m.perm = at, at += align16((size_t)SLOT_CHUNK * slot_byte_stride(N));
  m.source = at, at += align16((size_t)SLOT_CHUNK * slot_int_stride(receivers) * 2);
  m.dur = at, at += SLOT_CHUNK * 4;
  m.bad = at, at += 4;
  m.bytes = at;
  return m;
}

// SOURCES: start and length are computed (for the sources of this CTA's block); otherwise they are read back.
// RECEIVERS: rows and offsets are computed (all sources in one CTA).
template <bool SOURCES, bool RECEIVERS>
__global__ void __launch_bounds__(1024) slots_kernel(const SlotArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  const int N = a.N, P = a.P;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, threads = blockDim.x;
  const int part = blockIdx.x % a.CS;          // stretch of the matchings
  const size_t b = blockIdx.x / a.CS;
  const int i0 = SOURCES && !RECEIVERS ? blockIdx.y * SLOT_BLOCK : 0;
  const int sources = SOURCES && !RECEIVERS ? min(SLOT_BLOCK, N - i0) : N;
  const SlotSmem at = slot_smem(N, SOURCES && !RECEIVERS ? SLOT_BLOCK : N, SOURCES, RECEIVERS ? N : 0);
  const int IS = slot_int_stride(SOURCES && !RECEIVERS ? SLOT_BLOCK : N), BS = slot_byte_stride(N);
  int2* pairs = reinterpret_cast<int2*>(smem + at.pairs);          // x used, y demand
  long long* received = reinterpret_cast<long long*>(smem + at.received);
  int* c_start = reinterpret_cast<int*>(smem + at.start);
  int* c_len = reinterpret_cast<int*>(smem + at.len);
  int* c_begins = reinterpret_cast<int*>(smem + at.begins);        // by receiver: length, then first row
  uint8_t* c_perm = smem + at.perm;
  short* c_source = reinterpret_cast<short*>(smem + at.source);    // by receiver; -1 where no source named it
  int* c_dur = reinterpret_cast<int*>(smem + at.dur);
  int* bad_flag = reinterpret_cast<int*>(smem + at.bad);

  const int32_t* D = a.demand + b * N * N;
  const uint8_t* perm = a.perm + b * a.K * N;
  const int32_t* dur = a.dur + b * a.K;
  const int count_in = a.count[b];
  bool bad = count_in < 0 || count_in > a.K;
  const int count = bad ? 0 : count_in;
  if (threadIdx.x == 0) *bad_flag = 0;
  if constexpr (SOURCES) {
    for (int q = threadIdx.x; q < sources * N; q += threads) {
      const int d = D[(size_t)i0 * N + q];
      bad |= d < 0;
      pairs[q] = make_int2(0, max(d, 0));
    }
  }
  if constexpr (RECEIVERS) {
    for (int j = threadIdx.x; j < N; j += threads) received[j] = 0;
  }
  const int chunks = (a.K + SLOT_CHUNK - 1) / SLOT_CHUNK;
  const int c_begin = (int)((long long)chunks * part / a.CS), c_end = (int)((long long)chunks * (part + 1) / a.CS);

  auto load_chunk = [&](int k0) {
    const int used_k = min(SLOT_CHUNK, count - k0);                // matchings of the chunk that count (may be negative)
    for (int q = threadIdx.x; q < SLOT_CHUNK * N; q += threads) {
      const int kk = q / N, i = q - kk * N;
      if (kk < used_k) c_perm[kk * BS + i] = perm[(size_t)k0 * N + q];
      if constexpr (RECEIVERS) c_source[kk * IS + i] = -1, c_begins[kk * IS + i] = 0;
    }
    if (threadIdx.x < SLOT_CHUNK) {
      const int d = (int)threadIdx.x < used_k ? dur[k0 + threadIdx.x] : 0;
      bad |= d < 0;
      c_dur[threadIdx.x] = max(d, 0);
    }
  };
  // a warp per source, a lane per matching; keep = false: only the pairs' used tokens move on
  auto walk_sources = [&](int k0, bool keep) {
    const bool live = k0 + lane < count;
    for (int i = warp; i < sources; i += warps) {
      int dest = live ? c_perm[lane * BS + i0 + i] : 0;
      const bool ok = live && dest < N;
      bad |= live && dest >= N;
      dest = ok ? dest : 0;
      const int d = ok ? c_dur[lane] : 0;
      const unsigned peers = __match_any_sync(FULL, ok ? dest : -1 - lane);
      long long before = 0;                                        // carried by earlier matchings of the chunk
      if (__any_sync(FULL, (peers & (peers - 1)) != 0)) {
#pragma unroll 4
        for (int s = 0; s < 31; ++s) {
          const int v = __shfl_sync(FULL, d, s);
          if (s < lane && ((peers >> s) & 1u)) before += v;
        }
      }
      const int2 p = ok ? pairs[MS_AT(i * N + dest, sources * N)] : make_int2(0, 0);
      const int first = (int)min((long long)p.y, p.x + before);
      const int len = min(p.y - first, d);
      __syncwarp();
      if (ok && (peers >> lane) == 1u) pairs[MS_AT(i * N + dest, sources * N)].x = first + len;
      __syncwarp();
      if (keep) {
        c_start[lane * IS + i] = first;
        c_len[lane * IS + i] = len;
        if constexpr (RECEIVERS) {
          if (ok) c_begins[lane * IS + dest] = len, c_source[lane * IS + dest] = (short)i;
        }
      }
    }
  };

  if constexpr (SOURCES && RECEIVERS) {
    if (a.CS > 1) {
      // What the stretches before this one have carried: every CTA first walks its own stretch alone, then adds up its
      // predecessors' figures (used = min(D, sum): a cut sum of what was cut before is the cut sum).
      __syncthreads();
      for (int c = c_begin; c < c_end && c * SLOT_CHUNK < count && part + 1 < a.CS; ++c) {
        load_chunk(c * SLOT_CHUNK);
        __syncthreads();
        walk_sources(c * SLOT_CHUNK, false);
        __syncthreads();
      }
      cluster_sync_all();
      constexpr int HELD = 16 * 1024 / 1024;                       // pairs per thread: N * N / threads with 1024 threads
      int held[HELD];
#pragma unroll
      for (int h = 0; h < HELD; ++h) {
        const int q = threadIdx.x + h * threads;
        long long sum = 0;
        if (q < N * N) {
          for (int c = 0; c < part; ++c) sum += *map_to_cta(&pairs[q].x, c);
          sum = min(sum, (long long)pairs[q].y);
        }
        held[h] = (int)sum;
      }
      cluster_sync_all();
#pragma unroll
      for (int h = 0; h < HELD; ++h) {
        const int q = threadIdx.x + h * threads;
        if (q < N * N) pairs[q].x = held[h];
      }
      __syncthreads();
      for (int j = threadIdx.x; j < N; j += threads) {
        long long sum = 0;
        for (int i = 0; i < N; ++i) sum += pairs[i * N + j].x;
        received[j] = sum;
      }
    }
  }

  for (int c = c_begin; c < c_end; ++c) {
    const int k0 = c * SLOT_CHUNK, held = min(SLOT_CHUNK, a.K - k0);
    __syncthreads();
    load_chunk(k0);
    __syncthreads();
    if constexpr (SOURCES) {
      walk_sources(k0, true);
    } else {
      for (int q = threadIdx.x; q < held * N; q += threads) {
        const int kk = q / N, i = q - kk * N;
        const size_t g = (b * a.K + k0) * N + q;
        const int len = a.length[g];
        c_start[kk * IS + i] = a.start[g];
        const int dest = k0 + kk < count ? c_perm[kk * BS + i] : N;
        bad |= k0 + kk < count && dest >= N;
        if (dest < N) c_begins[kk * IS + dest] = len, c_source[kk * IS + dest] = (short)i;
      }
    }
    __syncthreads();
    if constexpr (RECEIVERS) {
      const int k = k0 + lane;
      for (int j = warp; j < N; j += warps) {
        const int len = c_begins[lane * IS + j], i = c_source[lane * IS + j];
        bad |= k < count && i < 0;                                 // no source: another receiver has two
        int incl = len;
        bool over = false;                                         // lengths are < 2^31: the sum of 32 may pass that
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int v = __shfl_up_sync(FULL, incl, o);
          if (lane >= o) {
            over |= incl > 0x7fffffff - v;
            incl = (int)((unsigned)incl + (unsigned)v) & 0x7fffffff;
          }
        }
        const long long run = received[j];
        const int total = __shfl_sync(FULL, incl, 31);
        over |= run + incl > 0x7fffffffLL;
        bad |= over;
        const int begins = over ? 0 : (int)(run + incl - len);
        __syncwarp();
        if (lane == 0) received[j] = min(run + total, 0x7fffffffLL);
        c_begins[lane * IS + j] = k < count ? begins : 0;
        if (a.offsets != nullptr && lane < held) {
          int32_t* to = a.offsets + (b * N + j) * ((size_t)a.K * P + 1) + (size_t)k * P;
          if (k < count && i >= 0) {
            const int32_t* share = a.counts + (b * N + i) * ((size_t)N * P) + (size_t)j * P;
            const int first = c_start[lane * IS + i];
            long long ahead = 0;
            for (int e = 0; e < P; ++e) {
              to[e] = begins + (int)max(0LL, min(ahead - first, (long long)len));
              const int v = share[e];
              bad |= v < 0;
              ahead += v;
            }
            bad |= ahead != D[(size_t)i * N + j];
          } else {
            for (int e = 0; e < P; ++e) to[e] = begins;
          }
        }
      }
      __syncthreads();
    }
    for (int q = threadIdx.x; q < held * sources; q += threads) {
      const int kk = q / sources, i = q - kk * sources;
      const size_t g = (b * a.K + k0 + kk) * N + i0 + i;
      const bool live = k0 + kk < count;
      if constexpr (SOURCES) {
        a.start[g] = live ? c_start[kk * IS + i] : 0;
        a.length[g] = live ? c_len[kk * IS + i] : 0;
      }
      if constexpr (RECEIVERS) {
        const int dest = live ? min((int)c_perm[kk * BS + i], N - 1) : 0;
        a.row[g] = live ? c_begins[kk * IS + dest] : 0;
      }
    }
  }
  if constexpr (RECEIVERS) {
    __syncthreads();
    if (part + 1 == a.CS) {
      for (int j = threadIdx.x; j < N; j += threads) {
        a.rows[b * N + j] = (int)received[j];
        if (a.offsets != nullptr) a.offsets[(b * N + j + 1) * ((size_t)a.K * P + 1) - 1] = (int)received[j];
      }
    }
  }
  if (bad) *bad_flag = 1;
  __syncthreads();
  if constexpr (!RECEIVERS) {
    if (threadIdx.x == 0 && *bad_flag) a.status[b] = MOESCHED_ST_BAD_INPUT;   // (the receivers' kernel completes it)
    return;
  } else {
    bool any = *bad_flag != 0;
    if (a.CS > 1) {
      cluster_sync_all();
      for (int c = 0; c < a.CS; ++c) any |= *map_to_cta(bad_flag, c) != 0;
      cluster_sync_all();                                          // nobody leaves while others read
    }
    if constexpr (!SOURCES) any |= a.status[b] != MOESCHED_ST_OK;
    __syncthreads();
    if (threadIdx.x == 0 && part == 0) a.status[b] = any ? MOESCHED_ST_BAD_INPUT : MOESCHED_ST_OK;
    if (any) {                                                     // a rejected schedule moves nothing
      const int k0 = c_begin * SLOT_CHUNK, k1 = min(a.K, c_end * SLOT_CHUNK);
      for (size_t q = (size_t)k0 * N + threadIdx.x; q < (size_t)k1 * N; q += threads) {
        const size_t g = b * a.K * N + q;
        a.start[g] = a.length[g] = a.row[g] = 0;
      }
      for (int j = threadIdx.x; j < N; j += threads) {
        if (part + 1 == a.CS) a.rows[b * N + j] = 0;
        if (a.offsets != nullptr) {
          int32_t* to = a.offsets + (b * N + j) * ((size_t)a.K * P + 1);
          for (size_t q = (size_t)k0 * P; q < (size_t)k1 * P + (part + 1 == a.CS); ++q) to[q] = 0;
        }
      }
    }
  }
}

cudaError_t run_slots(int B, int N, const int32_t* demand, int K, const uint8_t* perm, const int32_t* dur, const int32_t* count,
                      int P, const int32_t* counts, int32_t* start, int32_t* length, int32_t* row, int32_t* rows,
                      int32_t* offsets, int32_t* status, cudaStream_t stream) {
  SlotArgs a{N, K, P, 1, demand, perm, dur, count, counts, start, length, row, rows, offsets, status};
  const int threads = 32 * (N >= 32 ? 32 : N < 4 ? 4 : N);
  if (N <= SLOT_FUSED_N) {
    const auto kern = slots_kernel<true, true>;
    const size_t smem = slot_smem(N, N, true, N).bytes;
    if (cudaError_t e = permit_shared_memory(kern, smem); e != cudaSuccess) return e;
    kern<<<(unsigned)B, threads, smem, stream>>>(a);
    return cudaGetLastError();
  }
  cudaError_t e = cudaMemsetAsync(status, 0, (size_t)B * sizeof(int32_t), stream);
  if (e != cudaSuccess) return e;
  const auto by_source = slots_kernel<true, false>;
  const auto by_receiver = slots_kernel<false, true>;
  size_t smem = slot_smem(N, SLOT_BLOCK, true, 0).bytes;
  if ((e = permit_shared_memory(by_source, smem)) != cudaSuccess) return e;
  by_source<<<dim3((unsigned)B, (unsigned)((N + SLOT_BLOCK - 1) / SLOT_BLOCK)), threads, smem, stream>>>(a);
  if ((e = cudaGetLastError()) != cudaSuccess) return e;
  smem = slot_smem(N, N, false, N).bytes;
  if ((e = permit_shared_memory(by_receiver, smem)) != cudaSuccess) return e;
  by_receiver<<<(unsigned)B, threads, smem, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace moesched
