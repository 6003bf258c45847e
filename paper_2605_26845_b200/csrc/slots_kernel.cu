// Where the tokens of a schedule go: its replay against the demand, with the place of every transfer.
//
// With j = pi_k(i), used = tokens of the pair (i, j) that matchings before k have carried:
//   start  = min(D_ij, used),  length = min(D_ij - start, dur_k),  row = tokens that j has received before matching k,
//   offsets[j][k P + e] = row + (tokens of the transfer that are for experts of j below e); a pair's tokens lie by expert.
// A pair's transfers depend on one another only through `used`, a receiver's rows only through a running sum. So a CTA takes 32
// matchings at a time: a warp per source with a lane per matching (equal destinations among the 32 are summed by votes), then a warp
// per receiver with a lane per matching and a prefix sum over the lanes, then coalesced stores by matching. The pairs'
// `used` and demand are in shared memory. Bound by instructions and latency, not by bytes (1024 x 64 ranks x 64 matchings with
// offsets for four experts: 98 us, the bytes 32): a step's gathers, sums and stores depend on one another.
#include "common.cuh"

namespace moesched {

constexpr int SLOT_CHUNK = 32;         // matchings per step: one per lane
constexpr int SLOT_FUSED_N = 128;      // up to here the pairs of a whole matrix fit one CTA's shared memory
constexpr int SLOT_BLOCK = 64;         // sources per CTA above

struct SlotArgs {
  int N, K, P, parts;                  // parts: CTAs of a matrix, each with a stretch of the matchings
  unsigned per_n, per_sources;         // 2^22 / N and 2^22 / (sources of a CTA), rounded up (see slot_row)
  unsigned per_p;                      // 2^16 / P, rounded up
  bool words, quads, rows4;            // four destinations, four choices by expert, four pairs at a time
  const int32_t* demand;
  const uint8_t* perm;
  const int32_t* dur;
  const int32_t* count;
  const int32_t* counts;               // [B][N][N * P] or NULL
  int32_t *start, *length, *row, *rows, *offsets, *scratch, *status;
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

// Zeroes the outputs of matrix b for matchings k0 .. k1 - 1, and what stands behind the last.
__device__ void clear_schedule(const SlotArgs& a, size_t b, long long k0, long long k1) {
  const int N = a.N, P = a.P;
  for (size_t q = (size_t)k0 * N + threadIdx.x; q < (size_t)k1 * N; q += blockDim.x) {
    const size_t g = b * a.K * N + q;
    a.start[g] = a.length[g] = a.row[g] = 0;
  }
  for (int j = threadIdx.x; j < N; j += blockDim.x) {
    if (k1 == a.K) a.rows[b * N + j] = 0;
    if (a.offsets != nullptr) {
      int32_t* to = a.offsets + (b * N + j) * ((size_t)a.K * P + 1);
      for (size_t q = (size_t)k0 * P; q < (size_t)k1 * P + (k1 == a.K); ++q) to[q] = 0;
    }
  }
}

// SOURCES: start and length are computed (for the sources of this CTA's block); otherwise they are read back.
// RECEIVERS: rows and offsets are computed (all sources in one CTA).
// INSIDE: the choices by expert of a pair are fetched where its source is walked (32 destinations lie in the one or two KB of a source's
// row, 32 sources of a receiver in as many rows) and the starts within the transfer left for the receiver in shared memory, where
// that leaves room for two CTAs on an SM: 1024 x 64 ranks x 4 experts 104 us in place of 119 (98 with the pairs loaded four at a time).
// PARTS: few matrices, long schedules. What a stretch of the matchings carries of each pair is walked first, for itself (without
// RECEIVERS; into scratch[matrix][part][pair]); prefix_kernel turns that into what all stretches before it carry, min(D, sum), a cut
// sum of cut sums; then every stretch is done as a schedule of its own that begins there. 4 x 128 ranks x 2304 matchings: 61 us; with
// the stretches on the CTAs of a cluster, 16 at most, which exchange through shared memory, 119; in one CTA 1728.
template <bool SOURCES, bool RECEIVERS, bool PARTS, bool INSIDE>
__global__ void __launch_bounds__(1024) slots_kernel(const SlotArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  const int N = a.N, P = a.P;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, threads = blockDim.x;
  const int part = PARTS ? blockIdx.x % a.parts : 0;   // stretch of the matchings
  const size_t b = PARTS ? blockIdx.x / a.parts : blockIdx.x;
  const int i0 = SOURCES && !RECEIVERS && !PARTS ? blockIdx.y * SLOT_BLOCK : 0;
  const int sources = SOURCES && !RECEIVERS && !PARTS ? min(SLOT_BLOCK, N - i0) : N;
  const SlotSmem at = slot_smem(N, SOURCES && !RECEIVERS && !PARTS ? SLOT_BLOCK : N, SOURCES, RECEIVERS ? N : 0, blockDim.x >> 5,
                               INSIDE ? 0 : slot_staged(P), INSIDE ? SLOT_CHUNK * P : 0);
  const int IS = slot_int_stride(SOURCES && !RECEIVERS && !PARTS ? SLOT_BLOCK : N), BS = slot_byte_stride(N), PS = slot_int_stride(N);
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
    if (a.rows4) {
#pragma unroll 4
      for (int i = warp; i < sources; i += warps) {
        for (int j = 4 * lane; j < N; j += 128) {
          const int4 d = *reinterpret_cast<const int4*>(D + (size_t)(i0 + i) * N + j);
          bad |= (d.x | d.y | d.z | d.w) < 0;
          int2* to = pairs + i * PS + j;
          to[0] = make_int2(0, max(d.x, 0)), to[1] = make_int2(0, max(d.y, 0));
          to[2] = make_int2(0, max(d.z, 0)), to[3] = make_int2(0, max(d.w, 0));
        }
      }
    } else {
      for (int i = warp; i < sources; i += warps) {
        for (int j = lane; j < N; j += 32) {
          const int d = D[(size_t)(i0 + i) * N + j];
          bad |= d < 0;
          pairs[i * PS + j] = make_int2(0, max(d, 0));
        }
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
  const int c_begin = (int)((long long)chunks * part / a.parts), c_end = (int)((long long)chunks * (part + 1) / a.parts);

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

  if constexpr (PARTS) {
    let_next_start();
    int32_t* carried = a.scratch + (b * a.parts + part) * ((size_t)N * N);
    if constexpr (!RECEIVERS) {
      __syncthreads();
      for (int c = c_begin; c < c_end && c * SLOT_CHUNK < count; ++c) {
        load_chunk(c * SLOT_CHUNK);
        __syncthreads();
        walk_sources(c * SLOT_CHUNK, false);
        __syncthreads();
      }
      for (int i = warp; i < N; i += warps)
        for (int j = lane; j < N; j += 32) carried[i * N + j] = pairs[i * PS + j].x;
      return;                                                      // (what is wrong is found again)
    } else {
      wait_for_previous();
      __syncthreads();
      if (a.rows4) {
#pragma unroll 4
        for (int i = warp; i < N; i += warps)
          if (4 * lane < N) {
            const int4 u = *reinterpret_cast<const int4*>(carried + i * N + 4 * lane);
            int2* to = pairs + i * PS + 4 * lane;
            to[0].x = u.x, to[1].x = u.y, to[2].x = u.z, to[3].x = u.w;
          }
      } else {
        for (int i = warp; i < N; i += warps)
          for (int j = lane; j < N; j += 32) pairs[i * PS + j].x = carried[i * N + j];
      }
      __syncthreads();
      for (int q = threadIdx.x; q < N * (threads / N); q += threads) {
        const int j = q % N, step = threads / N;
        unsigned long long sum = 0;
        for (int i = q / N; i < N; i += step) sum += (unsigned)pairs[i * PS + j].x;
        atomicAdd(reinterpret_cast<unsigned long long*>(received + j), sum);
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
      if constexpr (PARTS) next = meet(warp);
      for (int j = warp; j < N; j += warps) {
        Arrival now;
        if constexpr (PARTS) now = next, next = meet(j + warps);
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
    if (part + 1 == a.parts) {
      for (int j = threadIdx.x; j < N; j += threads) {
        a.rows[b * N + j] = (int)received[j];
        if (a.offsets != nullptr) a.offsets[(b * N + j + 1) * ((size_t)a.K * P + 1) - 1] = (int)received[j];
      }
    }
  }
  if (bad) *bad_flag = 1;
  __syncthreads();
  if constexpr (!RECEIVERS || PARTS) {
    if (threadIdx.x == 0 && *bad_flag) a.status[b] = MOESCHED_ST_BAD_INPUT;   // (another kernel completes it)
  } else {
    const bool any = *bad_flag != 0 || (!SOURCES && a.status[b] != MOESCHED_ST_OK);
    __syncthreads();
    if (threadIdx.x == 0) a.status[b] = any ? MOESCHED_ST_BAD_INPUT : MOESCHED_ST_OK;
    if (any) clear_schedule(a, b, 0, a.K);
  }
}

// See PARTS. A thread per pair; and the status that the stretches may then spoil.
__global__ void __launch_bounds__(256) prefix_kernel(const SlotArgs a) {
  let_next_start();
  wait_for_previous();
  const size_t b = blockIdx.x, pairs = (size_t)a.N * a.N;
  const int q = blockIdx.y * 256 + threadIdx.x;
  if (q == 0) a.status[b] = MOESCHED_ST_OK;
  if (q >= (int)pairs) return;
  const unsigned most = (unsigned)max(a.demand[b * pairs + q], 0);
  int32_t* at = a.scratch + b * a.parts * pairs + q;
  unsigned run = 0;
  constexpr int AHEAD = 16;
  for (int p0 = 0; p0 < a.parts; p0 += AHEAD) {
    int v[AHEAD];
#pragma unroll
    for (int p = 0; p < AHEAD; ++p) v[p] = p0 + p < a.parts ? at[(p0 + p) * pairs] : 0;
#pragma unroll
    for (int p = 0; p < AHEAD; ++p) {
      if (p0 + p < a.parts) at[(p0 + p) * pairs] = (int)run;
      run = min(run + (unsigned)v[p], most);
    }
  }
}
// A rejected schedule moves nothing, whichever stretch was wrong.
__global__ void __launch_bounds__(256) clear_kernel(const SlotArgs a) {
  wait_for_previous();
  const size_t b = blockIdx.x / a.parts;
  const int part = blockIdx.x % a.parts;
  if (a.status[b] != MOESCHED_ST_OK) clear_schedule(a, b, (long long)a.K * part / a.parts, (long long)a.K * (part + 1) / a.parts);
}

template <typename Kernel>
static cudaError_t launch_slots(Kernel kern, const SlotArgs& a, dim3 grid, int threads, size_t smem, bool early, cudaStream_t stream) {
  if (cudaError_t e = permit_shared_memory(kern, smem); e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr = start_early();
  cfg.attrs = &attr;
  cfg.numAttrs = early ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kern, a);
}

// Stretches of the matchings for a CTA each: with fewer matrices than half of the SMs and schedules of eight steps and more, as many
// as fill the GPU once, of two steps at least. 1: a CTA does all of a schedule.
static int slot_parts(int B, int N, int K) {
  const long long chunks = (K - 1) / SLOT_CHUNK + 1, sms = sm_count();
  if (N > SLOT_FUSED_N || chunks < 8 || B < 1 || 2LL * B > sms) return 1;
  const long long fill = (sms + B - 1) / B;
  return (int)(fill < chunks / 2 ? fill : chunks / 2);
}
size_t slots_scratch_bytes(int B, int N, int K) {
  const int parts = slot_parts(B, N, K);
  return parts > 1 ? (size_t)B * parts * N * N * sizeof(int32_t) : 0;
}

cudaError_t run_slots(int B, int N, const int32_t* demand, int K, const uint8_t* perm, const int32_t* dur, const int32_t* count,
                      int P, const int32_t* counts, int32_t* start, int32_t* length, int32_t* row, int32_t* rows,
                      int32_t* offsets, int32_t* scratch, int32_t* status, cudaStream_t stream) {
  if (offsets == nullptr) P = 0;
  SlotArgs a{N, K, P, 1, slot_reciprocal(N), slot_reciprocal(SLOT_BLOCK), P > 0 ? (65536u + P - 1) / P : 0, N % 4 == 0 && (reinterpret_cast<uintptr_t>(perm) & 3) == 0,
             P % 4 == 0 && (reinterpret_cast<uintptr_t>(counts) & 15) == 0,
             N % 4 == 0 && ((reinterpret_cast<uintptr_t>(demand) | reinterpret_cast<uintptr_t>(scratch)) & 15) == 0, demand, perm, dur, count, counts, start, length, row, rows,
             offsets, scratch, status};
  const int warps = N >= 16 ? 16 : N < 4 ? 4 : N;
  cudaError_t e;
  if (N <= SLOT_FUSED_N) {
    a.parts = scratch != nullptr ? slot_parts(B, N, K) : 1;
    if (a.parts > 1) {
      const int many = N >= 32 ? 32 : warps;
      const dim3 grid((unsigned)(B * a.parts));
      e = launch_slots(slots_kernel<true, false, true, false>, a, grid, 32 * many, slot_smem(N, N, true, 0, many, 0, 0).bytes, false, stream);
      if (e == cudaSuccess) e = launch_slots(prefix_kernel, a, dim3((unsigned)B, (unsigned)((N * N + 255) / 256)), 256, 0, true, stream);
      if (e == cudaSuccess)
        e = launch_slots(slots_kernel<true, true, true, false>, a, grid, 32 * many, slot_smem(N, N, true, N, many, slot_staged(P), 0).bytes, true, stream);
      return e == cudaSuccess ? launch_slots(clear_kernel, a, grid, 256, 0, true, stream) : e;
    }
    const size_t smem = slot_smem(N, N, true, N, warps, slot_staged(P), 0).bytes, more = slot_smem(N, N, true, N, warps, 0, SLOT_CHUNK * P).bytes;
    return P >= 1 && P <= SLOT_STAGED_P && 2 * (more + 1024) <= SMEM_LIMIT + 1024
               ? launch_slots(slots_kernel<true, true, false, true>, a, dim3((unsigned)B), 32 * warps, more, false, stream)
               : launch_slots(slots_kernel<true, true, false, false>, a, dim3((unsigned)B), 32 * warps, smem, false, stream);
  }
  if ((e = cudaMemsetAsync(status, 0, (size_t)B * sizeof(int32_t), stream)) != cudaSuccess) return e;
  e = launch_slots(slots_kernel<true, false, false, false>, a, dim3((unsigned)B, (unsigned)((N + SLOT_BLOCK - 1) / SLOT_BLOCK)), 32 * warps,
                   slot_smem(N, SLOT_BLOCK, true, 0, warps, 0, 0).bytes, false, stream);
  if (e != cudaSuccess) return e;
  return launch_slots(slots_kernel<false, true, false, false>, a, dim3((unsigned)B), 32 * warps,
                      slot_smem(N, N, false, N, warps, slot_staged(P), 0).bytes, false, stream);
}

}  // namespace moesched
