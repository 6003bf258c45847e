// Where the tokens of a schedule go: its replay against the demand, with the place of every transfer.
//
// With j = pi_k(i), used = tokens of the pair (i, j) that matchings before k have carried:
//   start  = min(D_ij, used),  length = min(D_ij - start, dur_k),  row = tokens that j has received before matching k,
//   offsets[j][k P + e] = row + (tokens of the transfer that are for experts of j below e); a pair's tokens lie by expert.
// A pair's transfers depend on one another only through `used`, a receiver's rows only through a running sum. So a CTA takes 32
// matchings at a time: a warp per source with a lane per matching (equal destinations among the 32 are summed by votes), then a warp
// per receiver with a lane per matching and a prefix sum over the lanes, then coalesced stores by matching. The pairs'
// `used` and demand are in shared memory. Bound by instructions and latency, not by bytes (1024 x 64 ranks x 64 matchings with
// offsets for four experts: 104 us, the bytes 32): a step's gathers, sums and stores depend on one another.
#include "common.cuh"

namespace moesched {

constexpr int SLOT_CHUNK = 32;         // matchings per step: one per lane
constexpr int SLOT_FUSED_N = 128;      // up to here the pairs of a whole matrix fit one CTA's shared memory
constexpr int SLOT_MAX_PARTS = 16;     // CTAs that share the matchings of one matrix (4 x 128 ranks x 2304: 118 us, with 8 CTAs 175)
constexpr int SLOT_BLOCK = 64;         // sources per CTA above

struct SlotArgs {
  int N, K, P, CS;                     // CS: CTAs of a cluster, each with a stretch of the matchings
  unsigned per_n, per_sources;         // 2^22 / N and 2^22 / (sources of a CTA), rounded up (see slot_row)
  unsigned per_p;                      // 2^16 / P, rounded up
  bool words, quads;                   // four destinations, four choices by expert at a time
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

// q / n for q < 32 n, n <= 256, with m = ceil(2^22 / n): the quotient is off by less than q / 2^22 < 1 / n
__host__ __device__ inline unsigned slot_reciprocal(int n) { return ((1u << 22) + n - 1) / n; }
__device__ __forceinline__ int slot_row(int q, unsigned m) { return (int)((unsigned)q * m >> 22); }
// offsets of a receiver that a warp collects before it stores them side by side (ints; more go out as they come)
constexpr int SLOT_STAGED_P = 8;
__host__ __device__ inline int slot_staged(int P) { return P <= SLOT_STAGED_P ? SLOT_CHUNK * P : 0; }

struct SlotSmem {
  size_t pairs, received, start, len, begins, perm, source, dur, bad, seen, staged, inside, bytes;
};
// `sources` in this CTA (with their pairs if it walks them), and `receivers` (all of them, or none)
__host__ __device__ inline SlotSmem slot_smem(int N, int sources, bool pairs, int receivers, int warps, int staged, int inside) {
  SlotSmem m;
  size_t at = 0;
  m.pairs = at, at += pairs ? align16((size_t)sources * slot_int_stride(N) * sizeof(int2)) : 0;
  m.received = at, at += align16((size_t)receivers * sizeof(long long));
  m.start = at, at += align16((size_t)SLOT_CHUNK * slot_int_stride(sources) * 4);
  m.len = at, at += align16((size_t)SLOT_CHUNK * slot_int_stride(sources) * 4);
  m.begins = at, at += align16((size_t)SLOT_CHUNK * slot_int_stride(receivers) * 4);
  m.perm = at, at += align16((size_t)SLOT_CHUNK * slot_byte_stride(N));
  m.source = at, at += align16((size_t)SLOT_CHUNK * slot_int_stride(receivers) * 2);
  m.dur = at, at += SLOT_CHUNK * 4;
  m.bad = at, at += 16;
  m.seen = at, at += pairs ? align16((size_t)warps * slot_byte_stride(N)) : 0;
  m.staged = at, at += (size_t)warps * staged * 4;
  m.inside = at, at += (size_t)receivers * inside * 4;
  m.bytes = at;
  return m;
}

// SOURCES: start and length are computed (for the sources of this CTA's block); otherwise they are read back.
// RECEIVERS: rows and offsets are computed (all sources in one CTA).
// SPLIT: a cluster of CTAs shares the matchings (one CTA to an SM: a receiver's gathers are then fetched one receiver ahead; with
// several CTAs to an SM that costs more than it hides, 138 in place of 123 us for 1024 x 64 ranks).
// INSIDE: the choices by expert of a pair are fetched where its source is walked (32 destinations lie in the one or two KB of a source's
// row, 32 sources of a receiver in as many rows) and the starts within the transfer left for the receiver in shared memory, where
// that leaves room for two CTAs on an SM: 1024 x 64 ranks x 4 experts 104 us in place of 119.
template <bool SOURCES, bool RECEIVERS, bool SPLIT, bool INSIDE>
__global__ void __launch_bounds__(1024) slots_kernel(const SlotArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  const int N = a.N, P = a.P;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, threads = blockDim.x;
  const int part = SPLIT ? blockIdx.x % a.CS : 0;   // stretch of the matchings
  const size_t b = SPLIT ? blockIdx.x / a.CS : blockIdx.x;
  const int i0 = SOURCES && !RECEIVERS ? blockIdx.y * SLOT_BLOCK : 0;
  const int sources = SOURCES && !RECEIVERS ? min(SLOT_BLOCK, N - i0) : N;
  const SlotSmem at = slot_smem(N, SOURCES && !RECEIVERS ? SLOT_BLOCK : N, SOURCES, RECEIVERS ? N : 0, blockDim.x >> 5,
                               INSIDE ? 0 : slot_staged(P), INSIDE ? SLOT_CHUNK * P : 0);
  const int IS = slot_int_stride(SOURCES && !RECEIVERS ? SLOT_BLOCK : N), BS = slot_byte_stride(N), PS = slot_int_stride(N);
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
    for (int i = warp; i < sources; i += warps) {
      for (int j = lane; j < PS; j += 32) {
        const int d = j < N ? D[(size_t)(i0 + i) * N + j] : 0;
        bad |= d < 0;
        pairs[i * PS + j] = make_int2(0, max(d, 0));
      }
    }
  }
  if constexpr (RECEIVERS) {
    for (int j = threadIdx.x; j < N; j += threads) received[j] = 0;
  }
  uint8_t* seen = smem + at.seen + warp * BS;                      // by receiver: a lane that has named it
  int* staged = reinterpret_cast<int*>(smem + at.staged) + warp * slot_staged(P);
  int* inside = reinterpret_cast<int*>(smem + at.inside);          // [receiver][matching][expert]
  const int chunks = (a.K - 1) / SLOT_CHUNK + 1;
  const int c_begin = (int)((long long)chunks * part / a.CS), c_end = (int)((long long)chunks * (part + 1) / a.CS);

  auto load_chunk = [&](int k0) {
    const int used_k = min(SLOT_CHUNK, count - k0);                // matchings of the chunk that count (may be negative)
    if (a.words) {
      const unsigned* from = reinterpret_cast<const unsigned*>(perm + (size_t)k0 * N);
      for (int q = threadIdx.x; 4 * q < used_k * N; q += threads) {
        const int kk = slot_row(4 * q, a.per_n), i = 4 * q - kk * N;
        *reinterpret_cast<unsigned*>(c_perm + kk * BS + i) = from[q];
      }
    } else {
      for (int q = threadIdx.x; q < used_k * N; q += threads) {
        const int kk = slot_row(q, a.per_n), i = q - kk * N;
        c_perm[kk * BS + i] = perm[(size_t)k0 * N + q];
      }
    }
    if constexpr (RECEIVERS)
      for (int q = threadIdx.x; q < SLOT_CHUNK * IS / 2; q += threads) reinterpret_cast<unsigned*>(c_source)[q] = FULL;   // -1, -1
    if (threadIdx.x < SLOT_CHUNK) {
      const int d = (int)threadIdx.x < used_k ? dur[k0 + threadIdx.x] : 0;
      bad |= d < 0;
      c_dur[threadIdx.x] = max(d, 0);
    }
  };
  const auto fetch = [&](const int32_t* at, bool live, int (&share)[4], int e0) {
    if (a.quads) {
      int4 v = make_int4(0, 0, 0, 0);
      if (live) v = *reinterpret_cast<const int4*>(at + e0);
      share[0] = v.x, share[1] = v.y, share[2] = v.z, share[3] = v.w;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) share[e] = live && e0 + e < P ? at[e0 + e] : 0;
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
      int share[4];
      const int32_t* shares = INSIDE ? a.counts + (b * N + i) * ((size_t)N * P) + (size_t)dest * P : nullptr;
      if constexpr (INSIDE) fetch(shares, ok, share, 0);
      // Do two lanes name one receiver? Each leaves its number there and looks whether it is still there. (Only then a
      // vote on equal destinations, which takes some 300 cycles for 32 different ones.)
      if (ok) seen[dest] = (uint8_t)lane;
      __syncwarp();
      unsigned peers = 1u << lane;
      long long before = 0;                                        // carried by earlier matchings of the chunk
      if (__any_sync(FULL, ok && *static_cast<volatile uint8_t*>(seen + dest) != lane)) {
        peers = __match_any_sync(FULL, ok ? dest : -1 - lane);
#pragma unroll 4
        for (int s = 0; s < 31; ++s) {
          const int v = __shfl_sync(FULL, d, s);
          if (s < lane && ((peers >> s) & 1u)) before += v;
        }
      }
      const int2 p = ok ? pairs[MS_AT(i * PS + dest, sources * PS)] : make_int2(0, 0);
      const int first = (int)min((long long)p.y, p.x + before);
      const int len = min(p.y - first, d);
      __syncwarp();
      if (ok && (peers >> lane) == 1u) pairs[MS_AT(i * PS + dest, sources * PS)].x = first + len;
      __syncwarp();
      if (keep) {
        c_start[lane * IS + i] = first;
        c_len[lane * IS + i] = len;
        if constexpr (RECEIVERS) {
          if (ok) c_begins[lane * IS + dest] = len, c_source[lane * IS + dest] = (short)i;
        }
        if constexpr (INSIDE) {
          int* to = inside + (dest * SLOT_CHUNK + lane) * P;
          long long ahead = -(long long)first;
          for (int e0 = 0; e0 < P; e0 += 4) {
            if (e0 > 0) fetch(shares, ok, share, e0);
            int v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              v[e] = (int)max(0LL, min(ahead, (long long)len));
              bad |= share[e] < 0;                                 // (0 behind the last expert)
              ahead += share[e];
            }
            if (!ok) continue;
            if (a.quads) {
              *reinterpret_cast<int4*>(to + e0) = make_int4(v[0], v[1], v[2], v[3]);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (e0 + e < P) to[e0 + e] = v[e];
            }
          }
          bad |= ok && ahead + first != p.y;
        }
      }
    }
  };

  if constexpr (SPLIT) {
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
    // every CTA adds up its share of the pairs for all CTAs, two pairs at a time
    const int quads = (N * PS + 1) / 2, q_begin = (int)((long long)quads * part / a.CS), q_end = (int)((long long)quads * (part + 1) / a.CS);
    for (int q = q_begin + threadIdx.x; q < q_end; q += threads) {
      unsigned lo = 0, hi = 0;
      for (int c0 = 0; c0 < a.CS; c0 += 4) {
        int4 v[4];
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (c0 + c < a.CS) v[c] = *reinterpret_cast<const int4*>(map_to_cta(&pairs[2 * q].x, c0 + c));
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          if (c0 + c >= a.CS) break;
          const unsigned more_lo = min(lo + (unsigned)v[c].x, (unsigned)v[c].y), more_hi = min(hi + (unsigned)v[c].z, (unsigned)v[c].w);
          *reinterpret_cast<int4*>(map_to_cta(&pairs[2 * q].x, c0 + c)) = make_int4((int)lo, v[c].y, (int)hi, v[c].w);
          lo = more_lo, hi = more_hi;
        }
      }
    }
    cluster_sync_all();
    for (int q = threadIdx.x; q < N * (threads / N); q += threads) {
      const int j = q % N, step = threads / N;
      unsigned long long sum = 0;
      for (int i = q / N; i < N; i += step) sum += (unsigned)pairs[i * PS + j].x;
      atomicAdd(reinterpret_cast<unsigned long long*>(received + j), sum);
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
        const int kk = slot_row(q, a.per_n), i = q - kk * N;
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
      // what a receiver's transfers need of memory is on its way while another's rows are summed
      struct Arrival {
        int i, pair, share[4];
        const int32_t* at;
      };
      const auto meet = [&](int j) {
        Arrival r;
        r.i = j < N ? c_source[lane * IS + j] : -1;
        const bool live = k < count && r.i >= 0;
        bad |= j < N && k < count && r.i < 0;                      // no source: another receiver has two
        r.pair = 0;
        r.at = nullptr;
        if (!INSIDE && a.offsets != nullptr) {
          r.at = a.counts + (b * N + (live ? r.i : 0)) * ((size_t)N * P) + (size_t)(live ? j : 0) * P;
          fetch(r.at, live, r.share, 0);
          if (live) r.pair = SOURCES ? pairs[r.i * PS + j].y : D[(size_t)r.i * N + j];
        }
        return r;
      };
      Arrival next;
      if constexpr (SPLIT) next = meet(warp);
      for (int j = warp; j < N; j += warps) {
        Arrival now;
        if constexpr (SPLIT) now = next, next = meet(j + warps);
        else now = meet(j);
        const bool live = k < count && now.i >= 0;
        const int len = live ? c_begins[lane * IS + j] : 0, first = live ? c_start[lane * IS + now.i] : 0;
        int incl = len;
        bool over = false;                                         // lengths are < 2^31: the sum of 32 may pass that
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int v = __shfl_up_sync(FULL, incl, o);
          if (lane >= o) {
            over |= incl > 0x7fffffff - v;
            incl = (int)(((unsigned)incl + (unsigned)v) & 0x7fffffffu);
          }
        }
        const long long run = received[j];
        const int total = __shfl_sync(FULL, incl, 31);
        over |= run + incl > 0x7fffffffLL;
        bad |= over;
        const int begins = over ? 0 : (int)(run + incl - len);
        __syncwarp();
        if (lane == 0) received[j] = min(run + total, 0x7fffffffLL);
        c_begins[lane * IS + j] = begins;
        if constexpr (INSIDE) {
          int32_t* to = a.offsets + (b * N + j) * ((size_t)a.K * P + 1) + (size_t)k0 * P;
          const int* from = inside + j * SLOT_CHUNK * P;
          const unsigned some = __ballot_sync(FULL, live);
          for (int q0 = 0; q0 < held * P; q0 += 32) {
            const int q = q0 + lane, kk = (int)((unsigned)q * a.per_p >> 16);    // (q < 32 P, P <= 8: exact)
            const int v = __shfl_sync(FULL, begins, kk & 31);
            if (q < held * P) to[q] = v + ((some >> kk & 1u) ? from[q] : 0);
          }
        } else if (a.offsets != nullptr) {
          int32_t* to = a.offsets + (b * N + j) * ((size_t)a.K * P + 1) + (size_t)k0 * P;
          long long ahead = 0;
          for (int e0 = 0; e0 < P; e0 += 4) {
            if (e0 > 0) fetch(now.at, live, now.share, e0);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              if (e0 + e >= P) break;
              const int v = begins + (int)max(0LL, min(ahead - first, (long long)len));
              if (P <= SLOT_STAGED_P) staged[lane * P + e0 + e] = v;
              else if (lane < held) to[lane * P + e0 + e] = v;
              bad |= now.share[e] < 0;
              ahead += now.share[e];
            }
          }
          bad |= live && ahead != now.pair;
          if (P <= SLOT_STAGED_P) {
            __syncwarp();
            for (int q = lane; q < held * P; q += 32) to[q] = staged[q];
            __syncwarp();
          }
        }
      }
      __syncthreads();
    }
    const unsigned per = sources == N ? a.per_n : sources == SLOT_BLOCK ? a.per_sources : slot_reciprocal(sources);
    for (int q = threadIdx.x; q < held * sources; q += threads) {
      const int kk = slot_row(q, per), i = q - kk * sources;
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
    if constexpr (SPLIT) {
      cluster_sync_all();
      for (int c = 0; c < a.CS; ++c) any |= *map_to_cta(bad_flag, c) != 0;
      cluster_sync_all();                                          // nobody leaves while others read
    }
    if constexpr (!SOURCES) any |= a.status[b] != MOESCHED_ST_OK;
    __syncthreads();
    if (threadIdx.x == 0 && part == 0) a.status[b] = any ? MOESCHED_ST_BAD_INPUT : MOESCHED_ST_OK;
    if (any) {                                                     // a rejected schedule moves nothing
      const long long k0 = (long long)c_begin * SLOT_CHUNK, k1 = min((long long)a.K, (long long)c_end * SLOT_CHUNK);
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

template <bool SOURCES, bool RECEIVERS, bool SPLIT, bool INSIDE>
static cudaError_t launch_slots(const SlotArgs& a, dim3 grid, int warps, size_t smem, cudaStream_t stream) {
  const auto kern = slots_kernel<SOURCES, RECEIVERS, SPLIT, INSIDE>;
  if (cudaError_t e = permit_shared_memory(kern, smem); e != cudaSuccess) return e;
  if (a.CS > 8)                                                    // beyond what every GPU of this kind must offer
    if (cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1); e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(32 * warps);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  if (SPLIT) {
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = a.CS;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
  }
  return cudaLaunchKernelEx(&cfg, kern, a);
}

cudaError_t run_slots(int B, int N, const int32_t* demand, int K, const uint8_t* perm, const int32_t* dur, const int32_t* count,
                      int P, const int32_t* counts, int32_t* start, int32_t* length, int32_t* row, int32_t* rows,
                      int32_t* offsets, int32_t* status, cudaStream_t stream) {
  if (offsets == nullptr) P = 0;
  SlotArgs a{N, K, P, 1, slot_reciprocal(N), slot_reciprocal(SLOT_BLOCK), P > 0 ? (65536u + P - 1) / P : 0, N % 4 == 0 && (reinterpret_cast<uintptr_t>(perm) & 3) == 0,
             P % 4 == 0 && (reinterpret_cast<uintptr_t>(counts) & 15) == 0, demand, perm, dur, count, counts, start, length, row, rows,
             offsets, status};
  int warps = N >= 16 ? 16 : N < 4 ? 4 : N;
  if (N <= SLOT_FUSED_N) {
    while (a.CS < SLOT_MAX_PARTS && (long long)B * a.CS * 2 <= sm_count() && K >= 2 * a.CS * SLOT_CHUNK) a.CS *= 2;
    if (a.CS > 1 && N >= 32) warps = 32;
    const size_t smem = slot_smem(N, N, true, N, warps, slot_staged(P), 0).bytes;
    if (a.CS > 1) return launch_slots<true, true, true, false>(a, dim3((unsigned)(B * a.CS)), warps, smem, stream);
    const size_t more = slot_smem(N, N, true, N, warps, 0, SLOT_CHUNK * P).bytes;
    return P >= 1 && P <= SLOT_STAGED_P && 2 * (more + 1024) <= SMEM_LIMIT + 1024
               ? launch_slots<true, true, false, true>(a, dim3((unsigned)B), warps, more, stream)
               : launch_slots<true, true, false, false>(a, dim3((unsigned)B), warps, smem, stream);
  }
  cudaError_t e = cudaMemsetAsync(status, 0, (size_t)B * sizeof(int32_t), stream);
  if (e != cudaSuccess) return e;
  e = launch_slots<true, false, false, false>(a, dim3((unsigned)B, (unsigned)((N + SLOT_BLOCK - 1) / SLOT_BLOCK)), warps,
                                slot_smem(N, SLOT_BLOCK, true, 0, warps, 0, 0).bytes, stream);
  if (e != cudaSuccess) return e;
  return launch_slots<false, true, false, false>(a, dim3((unsigned)B), warps, slot_smem(N, N, false, N, warps, slot_staged(P), 0).bytes, stream);
}

}  // namespace moesched
