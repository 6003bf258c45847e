// Products of a few rows with the weights of their experts: y = x W^T, or act(x Wg^T) * (x Wu^T), W in 16 bits, or in 4 bits
// with a scale for every group of weights along k, w = (q - 8) * scale.
//
// With a handful of rows the weights' bytes are all that counts. One CTA per SM stays; its warps (or groups of `split` warps, which
// share the k of an output and add up in shared memory in a fixed order) go through units of work by themselves: up to eight
// tokens of an expert and two tiles of 16 rows of its weights (of gate and up, or neighbours). Each warp has a ring of its own in
// shared memory that asynchronous copies keep filled, over the ends of units, with 64 bytes of each row and the tokens' x for
// the same k. The weights are the 16 rows of the matrix instruction (16 x 8 x 16) and the tokens its columns, so that a
// weight is unpacked once for all eight. Which k a lane holds is free as long as both operands agree on it: a lane takes
// neighbouring k. In 4 bits an instruction never mixes the groups of scales: the sum over one group is made in 32 bits of
// (q - 8) x, which 16-bit operands hold exactly, and scaled when it is added up.
// 16 bits: bound by the memory (16 rows of four experts of 7168 x 2048: 58 us for gate, up and down from a graph, 353 MB, 6.1 TB/s; 61 to 71
// call by call, other rows and weights every time). 4 bits: bound by
// the instructions that unpack, 5 (half) or 7 (bfloat16) for eight weights in the unit that shifts and masks, which issues every
// second cycle (61 rows of 32 experts, 2048 to 7168: 67 us, 3.7 TB/s).
#include "expert.cuh"

namespace moesched {

constexpr int FEW_WARPS = 16;
constexpr int FEW_ROWS = 8;         // tokens per pass over the weights
constexpr int FEW_TILE_ROWS = 32;   // rows of weights of a warp: two tiles of 16
constexpr int FEW_SLICE = 64;       // bytes of a row per step

struct FewArgs {
  int R, K, N, E, groups, split;
  const void *x, *w[2], *scale[2];
  const int32_t* offsets;
  void* y;
  float* sum[2];                    // the two products themselves, where they are wanted
  int32_t* status;
};

template <typename T>
__device__ __forceinline__ void mma16816(float (&c)[4], const unsigned (&a)[4], unsigned b0, unsigned b1) {
  if constexpr (std::is_same_v<T, __half>)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Four pairs (q0, q4), (q1, q5), (q2, q6), (q3, q7) of a word of eight 4-bit numbers, minus 8: a number under the leading bit
// of 2^7 (bfloat16) or 2^10 (half) is that power plus itself, and the difference of two such is exact. In half a number four bits up
// is 16 times itself there, and one fused operation takes it down; bfloat16 has too few bits for that.
__device__ __forceinline__ unsigned under(unsigned w, unsigned mask, unsigned lead) {
  unsigned v;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(v) : "r"(w), "r"(mask), "r"(lead));   // (w & mask) | lead
  return v;
}
template <typename T>
__device__ __forceinline__ void unpack4(unsigned w, unsigned (&v)[4]) {
  if constexpr (std::is_same_v<T, __half>) {
    const __half2 eight = __halves2half2(__ushort_as_half(0x6408), __ushort_as_half(0x6408));       // 2^10 + 8
    const __half2 sixteenth = __float2half2_rn(0.0625f), down = __float2half2_rn(-72.0f);           // (2^10 + 16 q) / 16 - 72 = q - 8
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const unsigned u = w >> (8 * q), lo = under(u, 0x000f000fu, 0x64006400u), hi = under(u, 0x00f000f0u, 0x64006400u);
      const __half2 d = __hsub2(*reinterpret_cast<const __half2*>(&lo), eight);
      const __half2 s = __hfma2(*reinterpret_cast<const __half2*>(&hi), sixteenth, down);
      v[2 * q] = *reinterpret_cast<const unsigned*>(&d);
      v[2 * q + 1] = *reinterpret_cast<const unsigned*>(&s);
    }
  } else {
    const unsigned eight = 0x43084308u;                                                             // 2^7 + 8
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const unsigned u = under(w >> (4 * q), 0x000f000fu, 0x43004300u);
      const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&u), *reinterpret_cast<const __nv_bfloat162*>(&eight));
      v[q] = *reinterpret_cast<const unsigned*>(&d);
    }
  }
}

// `bytes` of the 16 (4) are read, the rest is zero
__device__ __forceinline__ void copy16(unsigned dst, const void* src, unsigned bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
// (kept in L1: the warps of a CTA are mostly at the same tokens)
__device__ __forceinline__ void copy16_near(unsigned dst, const void* src, unsigned bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy4(unsigned dst, const void* src, unsigned bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

// GROUP: weights per scale, 0 for weights in 16 bits
template <int GROUP>
struct FewShape {
  static constexpr bool Q4 = GROUP != 0;
  static constexpr int BLOCK = FEW_SLICE * 8 / (Q4 ? 4 : 16);     // k per step of a warp: 128 or 32
  static constexpr int PIECES = Q4 ? BLOCK / (Q4 ? GROUP : 1) : 1;   // stretches of k that four lanes multiply together
  static constexpr int EACH = BLOCK / 4 / PIECES;                 // neighbouring k of a lane in a stretch
  static constexpr int WORDS = Q4 ? EACH / 8 : EACH / 2;          // 32-bit words of weights of a lane in a stretch
  static constexpr int LOADS = BLOCK / 32;                        // 16-byte parts of x of a lane in a step
  static constexpr int SCALE_WORDS = Q4 ? PIECES / 2 + 1 : 0;     // 32-bit words that cover a row's scales, which may begin within one
  static constexpr int X_AT = FEW_TILE_ROWS * FEW_SLICE, SCALE_AT = X_AT + LOADS * 512;
  static constexpr int STAGE = SCALE_AT + FEW_TILE_ROWS * 4 * SCALE_WORDS;
  // steps in a ring; the bytes of weights on their way to an SM are then 64 (group 32) to 128 KB, where the memory's rate
  // times its latency is some 43 KB
  static constexpr int STAGES = !Q4 ? 4 : GROUP == 32 ? 2 : 3;
  static constexpr int RING = FEW_WARPS * STAGES * STAGE;
  // the sums of the warps of a team: two sets where they fit, so that a warp need not wait until the others have read its last
  static constexpr int SUM_SETS = Q4 ? 1 : 2;
  static constexpr int SET = FEW_WARPS * 2 * FEW_ROWS * 16;       // floats: [warp][tile][token][16]
  static constexpr int SUMS = SUM_SETS * SET * 4;
  static constexpr int SMEM = RING + SUMS + MOESCHED_MAX_EXPERTS * 2 + 64;
  static_assert(SMEM <= SMEM_LIMIT, "shared memory");
  static_assert(RING >= MOESCHED_MAX_EXPERTS * 8, "units of the experts lie in the rings at first");
};

// Place of 16-byte part c of a row's slice: the rows that lanes read together lie in different banks, whether a lane reads 16
// bytes (two rows at once), 8 (four rows) or 4 (eight rows).
__device__ __forceinline__ int few_place(int row, int c) {
  return row * FEW_SLICE + ((c ^ ((row & 2) | (row >> 2 & 1))) << 4);
}

// Where a warp is: unit = (expert, outputs, eight of its rows), and the step in it
struct FewCursor {
  long long left;                 // units after this one
  int expert, passes, tile, pass; // expert: its number among those with rows; passes: eights of rows
  int row, rows;                  // row of this lane's token (lane / 4), or -1; rows of the expert
};

template <typename T, int GROUP, bool GATED, int ACT>
__global__ void __launch_bounds__(32 * FEW_WARPS, 1) few_kernel(const FewArgs a) {
  using Shape = FewShape<GROUP>;
  constexpr bool Q4 = Shape::Q4;
  constexpr int BLOCK = Shape::BLOCK, PIECES = Shape::PIECES, EACH = Shape::EACH, WORDS = Shape::WORDS, LOADS = Shape::LOADS,
                SCALE_WORDS = Shape::SCALE_WORDS, STAGE = Shape::STAGE, STAGES = Shape::STAGES;
  extern __shared__ __align__(16) unsigned char smem[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned char* ring = smem + warp * (STAGES * STAGE);
  long long* unit_end = reinterpret_cast<long long*>(smem);                       // (in the rings, before they are used)
  float* sums = reinterpret_cast<float*>(smem + Shape::RING);                     // [warp][tile][token][16]
  uint16_t* busy = reinterpret_cast<uint16_t*>(smem + Shape::RING + Shape::SUMS); // the experts with rows
  long long* scan = reinterpret_cast<long long*>(sums);
  const int R = a.R, K = a.K, N = a.N;
  const int split = a.split, part = warp % split;
  constexpr int OUTPUTS = GATED ? 16 : 32;                // of a warp
  const int tiles = (N + OUTPUTS - 1) / OUTPUTS;
  const int gr = lane >> 2, t = lane & 3;

  let_next_start();
  // experts with rows, and the units up to the end of each
  bool bad = false;
  int experts = 0;
  long long units = 0;
  for (int e0 = 0; e0 < a.E; e0 += 32 * FEW_WARPS) {
    const int e = e0 + threadIdx.x;
    long long have = 0;
    if (e < a.E)
      for (long long g = e; g < a.groups; g += a.E) {
        const int2 span = make_int2(a.offsets[g], a.offsets[g + 1]);
        if (rows_in_order(span, R)) have += span.y - span.x;
        else bad = true;
      }
    // units in the upper bits, experts in the lower ten and one
    long long incl = have > 0 ? ((have + FEW_ROWS - 1) / FEW_ROWS * tiles) << 11 | 1 : 0;
    const long long own = incl;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long v = __shfl_up_sync(FULL, incl, o);
      if (lane >= o) incl += v;
    }
    if (lane == 31) scan[warp] = incl;
    __syncthreads();
    long long before = 0, all = 0;
    for (int w = 0; w < FEW_WARPS; ++w) {
      before += w < warp ? scan[w] : 0;
      all += scan[w];
    }
    __syncthreads();
    incl += before;
    if (own != 0) {
      const int at = experts + (int)(incl & 2047) - 1;
      busy[MS_AT(at, MOESCHED_MAX_EXPERTS)] = (uint16_t)e;
      unit_end[MS_AT(at, MOESCHED_MAX_EXPERTS)] = units + (incl >> 11);
    }
    experts += (int)(all & 2047);
    units += all >> 11;
  }
  if (__syncthreads_or(bad)) {                            // (every CTA looks at all groups)
    wait_for_previous();
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = MOESCHED_ST_BAD_INPUT;
    fill(a.y, (size_t)R * N * 2, NANS, blockIdx.x, gridDim.x);
    if (a.sum[0] != nullptr) {
      fill(a.sum[0], (size_t)R * N * 4, NANS, blockIdx.x, gridDim.x);
      fill(a.sum[1], (size_t)R * N * 4, NANS, blockIdx.x, gridDim.x);
    }
    return;
  }

  // this warp's units
  const int teams = gridDim.x * (FEW_WARPS / split), team = blockIdx.x * (FEW_WARPS / split) + warp / split;
  // (divisions of 64 bits take a microsecond here, together; those of 32 are for all but calls that take long anyway)
  const bool few = units * teams < 1LL << 32;
  const auto share = [&](int q) {
    return few ? (long long)((unsigned)units * (unsigned)q / (unsigned)teams) : units * q / teams;
  };
  const long long first = share(team), mine = share(team + 1) - first;
  // rows of the expert, and of them the one of this lane's token in eight number `pass`
  const auto find_rows = [&](FewCursor& c) {
    const int e = busy[c.expert], skip = c.pass * FEW_ROWS;
    c.row = -1;
    if (a.groups == a.E) {                                // one group each: nothing to look for, which is a microsecond less
      const int2 span = rows_of_group(a.offsets, e, R);
      c.rows = span.y - span.x;
      c.passes = (c.rows + FEW_ROWS - 1) / FEW_ROWS;
      if (skip + gr < c.rows) c.row = span.x + skip + gr;
      return;
    }
    // (the groups are in order: no sum passes R, which is 2^30 at most)
    unsigned seen = 0;
    for (long long g0 = e; g0 < a.groups; g0 += 32LL * a.E) {
      const long long g = g0 + (long long)lane * a.E;
      const int2 span = g < a.groups ? rows_of_group(a.offsets, (int)g, R) : make_int2(0, 0);
      unsigned incl = span.y - span.x;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const unsigned v = __shfl_up_sync(FULL, incl, o);
        if (lane >= o) incl += v;
      }
      const int token = skip + gr - (int)seen;            // of this lane, from this round's first row on
      int at = 0;                                         // groups that end before it
#pragma unroll
      for (int o = 16; o > 0; o >>= 1)
        if ((int)__shfl_sync(FULL, incl, at + o - 1) <= token) at += o;
      const int end = (int)__shfl_sync(FULL, incl, at), row = __shfl_sync(FULL, span.y, at) - (end - token);
      if (token >= 0 && token < end) c.row = row;
      seen += __shfl_sync(FULL, incl, 31);
    }
    c.rows = (int)seen;
    c.passes = (c.rows + FEW_ROWS - 1) / FEW_ROWS;
  };
  FewCursor get = {};                                     // of the copies; `put_` of the products
  get.left = mine - 1;
  if (mine > 0) {
    int lo = 0, hi = experts - 1;
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (unit_end[mid] > first) hi = mid;
      else lo = mid + 1;
    }
    get.expert = lo;
    const long long begin = lo > 0 ? unit_end[lo - 1] : 0;
    find_rows(get);
    const long long into = first - begin;
    if (few) {
      get.tile = (int)((unsigned)into / (unsigned)get.passes);
      get.pass = (int)into - get.tile * get.passes;
    } else {
      get.tile = (int)(into / get.passes);
      get.pass = (int)(into % get.passes);
    }
    if (get.pass > 0) find_rows(get);
  }
  __syncthreads();                                        // the rings are the warps' own from here on
  wait_for_previous();                                    // x may come from the kernel before this one
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = MOESCHED_ST_OK;
  if (mine <= 0) return;
  const auto next_unit = [&](FewCursor& c) {
    --c.left;
    if (++c.pass == c.passes) {
      c.pass = 0;
      if (++c.tile == tiles) c.tile = 0, ++c.expert;
      else if (c.passes == 1) return;                     // the same rows
    }
    find_rows(c);
  };

  const size_t row_bytes = Q4 ? (size_t)K / 2 : (size_t)K * 2;
  const int steps = ((K + BLOCK - 1) / BLOCK + split - 1) / split;
  const char* wp[2];                                      // row lane / 4 of the two tiles, this lane's 16 bytes of the step
  const T* sp = nullptr;                                  // scales of row `lane` of both
  const T* xp = nullptr;                                  // this lane's token, its first k of the step
  unsigned valid = 0;                                     // rows lane / 4 and lane / 4 + 8 of the two tiles
  bool whole = false;                                     // all rows of the tiles exist
  int get_k = 0;                                          // first k of the step
  const auto aim = [&]() {
    const int e = busy[get.expert], n0 = get.tile * OUTPUTS;
    valid = 0;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const int n = n0 + (GATED ? 0 : 16 * m) + gr;
      wp[m] = static_cast<const char*>(a.w[GATED ? m : 0]) + ((size_t)e * N + min(n, N - 1)) * row_bytes + part * FEW_SLICE + t * 16;
      valid |= (n < N ? 1u : 0u) << (2 * m) | (n + 8 < N ? 2u : 0u) << (2 * m);
    }
    whole = n0 + OUTPUTS <= N;
    if constexpr (Q4) {
      const int n = n0 + (GATED ? lane & 15 : lane);
      sp = static_cast<const T*>(a.scale[GATED ? lane >> 4 : 0]) + ((size_t)e * N + min(n, N - 1)) * (K / (Q4 ? GROUP : 1));
    }
    get_k = part * BLOCK;
    xp = static_cast<const T*>(a.x) + (size_t)max(get.row, 0) * K + get_k + t * EACH;
  };
  aim();
  int get_step = 0, get_stage = 0;
  const auto issue = [&]() {                              // the next step's copies; a group of them in any case
    if (get.left >= 0) {
      const unsigned at = smem_addr(ring) + get_stage * STAGE, w_at = at + few_place(gr, t), x_at = at + Shape::X_AT + lane * 16;
      if (whole && get_k + BLOCK <= K) {
        const unsigned some = get.row >= 0 ? 16 : 0;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int r = 0; r < 2; ++r) copy16(w_at + (16 * m + 8 * r) * FEW_SLICE, wp[m] + (r ? 8 * row_bytes : 0), 16);
#pragma unroll
        for (int q = 0; q < LOADS; ++q) copy16_near(x_at + q * 512, xp + q / (EACH / 8) * 4 * EACH + q % (EACH / 8) * 8, some);
      } else {
        const bool in = get_k + t * (BLOCK / 4) < K;      // (this lane's 16 bytes of the rows)
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const bool ok = in && (valid >> (2 * m + r) & 1u);
            copy16(w_at + (16 * m + 8 * r) * FEW_SLICE, ok ? wp[m] + (r ? 8 * row_bytes : 0) : static_cast<const char*>(a.w[0]), ok ? 16 : 0);
          }
#pragma unroll
        for (int q = 0; q < LOADS; ++q) {
          const int o = q / (EACH / 8) * 4 * EACH + q % (EACH / 8) * 8;
          const bool ok = get.row >= 0 && get_k + t * EACH + o < K;
          copy16_near(x_at + q * 512, ok ? xp + o : static_cast<const T*>(a.x), ok ? 16 : 0);
        }
      }
      if constexpr (Q4) {
        const int s = get_k / (Q4 ? GROUP : 1), left = K / (Q4 ? GROUP : 1) - s;   // scales from here to the row's end
        const T* from = reinterpret_cast<const T*>(reinterpret_cast<uintptr_t>(sp + s) & ~(uintptr_t)3);
        const int back = (int)(sp + s - from);
#pragma unroll
        for (int q = 0; q < SCALE_WORDS; ++q) {
          const int have = left + back - 2 * q;
          copy4(at + Shape::SCALE_AT + (lane * SCALE_WORDS + q) * 4, have > 0 ? from + 2 * q : static_cast<const T*>(a.scale[0]),
                have > 1 ? 4 : have > 0 ? 2 : 0);
        }
      }
#pragma unroll
      for (int m = 0; m < 2; ++m) wp[m] += split * FEW_SLICE;
      xp += split * BLOCK;
      get_k += split * BLOCK;
      if (++get_stage == STAGES) get_stage = 0;
      if (++get_step == steps) {
        get_step = 0;
        if (get.left > 0) {
          next_unit(get);
          aim();
        } else {
          get.left = -1;
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };

  FewCursor use = get;
#pragma unroll 1
  for (int u = 0; u < STAGES - 1; ++u) issue();
  int stage = 0, set = 0;
  for (;;) {
    float acc[2][4];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int q = 0; q < 4; ++q) acc[m][q] = 0.0f;
    // where the scales of this lane's four rows are: in the upper half of a word if the number of the first is odd
    int scale_at[2][2] = {};
    if constexpr (Q4) {
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const size_t n = (size_t)busy[use.expert] * N + min(use.tile * OUTPUTS + (GATED ? 0 : 16 * m) + 8 * r + gr, N - 1);
          scale_at[m][r] = Shape::SCALE_AT + (16 * m + 8 * r + gr) * SCALE_WORDS * 4 + 2 * (int)(n * (K / (Q4 ? GROUP : 1)) + part * PIECES & 1);
        }
    }
    for (int i = 0; i < steps; ++i) {
      issue();
      asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
      __syncwarp();
      const unsigned char* at = ring + stage * STAGE;
      if (++stage == STAGES) stage = 0;
      if constexpr (Q4 && PIECES % 2 != 0) {              // with one scale a step their number changes parity from step to step
        if (i > 0 && split == 1) {
#pragma unroll
          for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int r = 0; r < 2; ++r) scale_at[m][r] ^= 2;
        }
      }
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        float sum[2][4];
        unsigned w[2][2][WORDS];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
#pragma unroll
          for (int q = 0; q < 4; ++q) sum[m][q] = Q4 ? 0.0f : acc[m][q];
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const int byte = (p * 4 + t) * WORDS * 4;     // of the lane's weights in the slice
            const unsigned char* from = at + few_place(16 * m + 8 * r + gr, byte >> 4) + (byte & 15);
            if constexpr (WORDS == 4) {
              const uint4 v = *reinterpret_cast<const uint4*>(from);
              w[m][r][0] = v.x, w[m][r][1] = v.y, w[m][r][2] = v.z, w[m][r][3] = v.w;
            } else if constexpr (WORDS == 2) {
              const uint2 v = *reinterpret_cast<const uint2*>(from);
              w[m][r][0] = v.x, w[m][r][1] = v.y;
            } else {
              w[m][r][0] = *reinterpret_cast<const unsigned*>(from);
            }
          }
        }
#pragma unroll
        for (int q = 0; q < EACH / 8; ++q) {
          uint4 v = *reinterpret_cast<const uint4*>(at + Shape::X_AT + ((p * (EACH / 8) + q) * 32 + lane) * 16);
          if constexpr (Q4)          // in the order of unpack4's pairs
            v = make_uint4(__byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632), __byte_perm(v.y, v.w, 0x5410),
                           __byte_perm(v.y, v.w, 0x7632));
#pragma unroll
          for (int m = 0; m < 2; ++m) {
            unsigned lo[4], hi[4];
            if constexpr (Q4) {
              unpack4<T>(w[m][0][q], lo);
              unpack4<T>(w[m][1][q], hi);
            } else {
#pragma unroll
              for (int c = 0; c < 4; ++c) lo[c] = w[m][0][4 * q + c], hi[c] = w[m][1][4 * q + c];
            }
            const unsigned f0[4] = {lo[0], hi[0], lo[1], hi[1]}, f1[4] = {lo[2], hi[2], lo[3], hi[3]};
            mma16816<T>(sum[m], f0, v.x, v.y);
            mma16816<T>(sum[m], f1, v.z, v.w);
          }
        }
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          float s[2] = {1.0f, 1.0f};
          if constexpr (Q4) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              s[r] = to_float(*reinterpret_cast<const T*>(at + scale_at[m][r] + 2 * p));
            }
          }
#pragma unroll
          for (int q = 0; q < 4; ++q) acc[m][q] = Q4 ? fmaf(s[q >> 1], sum[m][q], acc[m][q]) : sum[m][q];
        }
      }
      __syncwarp();
    }
    // lane (gr, t) has outputs gr, gr + 8 of the tokens 2t, 2t + 1
    float* to_sums = sums + set * Shape::SET + warp * (2 * FEW_ROWS * 16);
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int q = 0; q < 4; ++q) to_sums[(m * FEW_ROWS + 2 * t + (q & 1)) * 16 + gr + 8 * (q >> 1)] = acc[m][q];
    const int team_bar = 1 + warp / split, team_threads = 32 * split;
    if (split == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(team_bar), "r"(team_threads) : "memory");
    const float* team_sums = sums + set * Shape::SET + (warp - part) * (2 * FEW_ROWS * 16);
    for (int q = part * 32 + lane; q < FEW_ROWS * OUTPUTS; q += team_threads) {
      const int c = q % OUTPUTS, r = q / OUTPUTS, n = use.tile * OUTPUTS + c;
      const int row = __shfl_sync(FULL, use.row, r * 4 & 31);
      if (row < 0 || n >= N) continue;
      float v[2] = {0.0f, 0.0f};
#pragma unroll
      for (int m = 0; m < (GATED ? 2 : 1); ++m)
        for (int s = 0; s < split; ++s) v[m] += team_sums[((s * 2 + (GATED ? m : c >> 4)) * FEW_ROWS + r) * 16 + (c & 15)];
      const size_t to = (size_t)row * N + n;
      if constexpr (GATED) {
        if (a.sum[0] != nullptr) {
          a.sum[0][to] = v[0];
          a.sum[1][to] = v[1];
        }
        put(static_cast<T*>(a.y) + to, activation<ACT>(v[0]) * v[1]);
      } else {
        put(static_cast<T*>(a.y) + to, v[0]);
      }
    }
    if (use.left == 0) break;
    next_unit(use);
    // the sums are read before they are written again: with two sets, by the barrier of the next unit
    if constexpr (Shape::SUM_SETS == 2) set ^= 1;
    else if (split > 1) {
      __syncwarp();                                       // (lanes without a row to store may be ahead; a barrier is for whole warps)
      asm volatile("bar.sync %0, %1;" ::"r"(team_bar), "r"(team_threads) : "memory");
    }
    __syncwarp();
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
}

template <typename T, int GROUP, bool GATED, int ACT>
static cudaError_t launch_few(const FewArgs& a, bool early, cudaStream_t stream) {
  const auto kern = few_kernel<T, GROUP, GATED, ACT>;
  const size_t smem = FewShape<GROUP>::SMEM;
  if (cudaError_t e = permit_shared_memory(kern, smem); e != cudaSuccess) return e;
  const long long tiles = (a.N + (GATED ? 15 : 31)) / (GATED ? 16 : 32), teams = FEW_WARPS / a.split;
  const long long units = (a.R / FEW_ROWS + (a.E < a.R ? a.E : a.R)) * tiles, ctas = (units + teams - 1) / teams, sms = sm_count();
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(ctas < 1 ? 1 : ctas < sms ? ctas : sms));
  cfg.blockDim = dim3(32 * FEW_WARPS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr = start_early();
  cfg.attrs = &attr;
  cfg.numAttrs = early ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kern, a);
}
template <typename T, int GROUP>
static cudaError_t launch_few(const FewArgs& a, bool gated, int act, bool early, cudaStream_t stream) {
  if (!gated) return launch_few<T, GROUP, false, MOESCHED_ACT_SILU>(a, early, stream);
  if (act == MOESCHED_ACT_SILU) return launch_few<T, GROUP, true, MOESCHED_ACT_SILU>(a, early, stream);
  return launch_few<T, GROUP, true, MOESCHED_ACT_GELU>(a, early, stream);
}

cudaError_t run_few(int R, int K, int N, int E, int groups, int group, int dtype, int act, const void* x, const void* w,
                    const void* scale, const void* w_up, const void* scale_up, const int32_t* offsets, void* y, float* sum,
                    float* sum_up, int32_t* status, bool early, cudaStream_t stream) {
  FewArgs a{R, K, N, E, groups, 1, x, {w, w_up}, {scale, scale_up}, offsets, y, {sum, sum_up}, status};
  const bool gated = w_up != nullptr;
  // Warps share the k of an output only until half of the GPU's warps have a unit: every sharing costs a barrier and a sum (four
  // experts of 7168 x 2048 in 16 bits, 16 rows, from a graph: 60 us then, 58 now; until all have one 64, four each 73, a quarter of them 69).
  const long long units = (long long)(E < R ? E : R) * ((N + (gated ? 15 : 31)) / (gated ? 16 : 32));
  while (a.split < FEW_WARPS && 2 * units * a.split < (long long)FEW_WARPS * sm_count()) a.split *= 2;
  if (dtype == MOESCHED_BF16) {
    if (group == 0) return launch_few<__nv_bfloat16, 0>(a, gated, act, early, stream);
    if (group == 32) return launch_few<__nv_bfloat16, 32>(a, gated, act, early, stream);
    if (group == 64) return launch_few<__nv_bfloat16, 64>(a, gated, act, early, stream);
    return launch_few<__nv_bfloat16, 128>(a, gated, act, early, stream);
  }
  if (group == 0) return launch_few<__half, 0>(a, gated, act, early, stream);
  if (group == 32) return launch_few<__half, 32>(a, gated, act, early, stream);
  if (group == 64) return launch_few<__half, 64>(a, gated, act, early, stream);
  return launch_few<__half, 128>(a, gated, act, early, stream);
}

}  // namespace moesched
