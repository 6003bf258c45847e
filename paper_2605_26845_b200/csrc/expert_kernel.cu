// Gated feed-forward block of the experts on rows grouped by expert, and its backward pass: five products on the tensor
// cores, with what stands between them in their epilogues.
//
//   GLU      a = X Wg^T, u = X Wu^T                    -> h = act(a) u (and a, u for the backward pass)
//   DOWN     y = h Wd^T
//   DHIDDEN  dh = dY Wd                                -> h again, du = dh act(a), da = dh u act'(a)
//   DINPUT   dX = da Wg + du Wu                        (one contraction over 2 I)
//   DWEIGHT  dWg = da^T X, dWu = du^T X, dWd = dY^T h  (contractions over the rows of an expert)
//
// Persistent CTAs take tiles of 128 x 128 (GLU: 64 columns of a and the same 64 of u), or pairs of CTAs on two SMs tiles of
// 256 x 256, each with half of the rows of either operand: every byte that a pair fetches serves twice as many products. One warp fetches
// the operands with TMA, 64 deep, into a ring of stages; one thread (of a pair: of its first CTA) issues the matrix instructions, whose
// sums are in tensor memory, twice, so that eight warps empty one while the other fills; those warps turn what they
// read by way of shared memory, so that neighbouring lanes load and store neighbouring columns. Operands stay as they are in memory:
// where the contraction runs over the slower axis (Wd in DHIDDEN, Wg and Wu in DINPUT, everything in DWEIGHT) the instruction
// takes them transposed.
// Row tiles of the groups are laid out by a small kernel first (plan_kernel): a tile never spans two groups, what lies behind its
// group's last row is computed and not stored. In DWEIGHT the rows are the contraction: there the rows behind
// a group's last, up to the next multiple of 16, are zeroed in shared memory (0 x NaN would not be nothing).
// Single launches of eight experts, 4096 x 2048, 16384 rows: GLU 361 us (1.52 PFLOP/s, tensor cores busy 89 % of the cycles), DOWN 161,
// DHIDDEN 244 (60 %: it moves 1.0 GB beside its product, a and u in 32 bits among them), DINPUT 339 (93 %), DWEIGHT 563 (81 %), 1670 in all;
// back to back they take 1960 to 2300 a pass, as the clock falls to 1.3 to 1.5 GHz: what bounds the large products is the power.
#include <cuda.h>

#include <atomic>

#include "expert.cuh"

namespace moesched {

enum { GLU, DOWN, DHIDDEN, DINPUT, DWEIGHT };

constexpr int CTA_M = 128, CTA_N = 128, BK = 64;           // rows of the operands that a CTA fetches, and how deep
constexpr int STAGES = 6;
constexpr int A_BYTES = CTA_M * BK * 2, B_BYTES = CTA_N * BK * 2, STAGE_BYTES = A_BYTES + B_BYTES;
constexpr int EMPTIERS = 8;                                // warps that empty tensor memory: two for each quarter of its lanes
constexpr int GEMM_THREADS = 128 + 32 * EMPTIERS;
constexpr int BOX_BYTES = 64 * 64 * 2;                     // one box of B, and of a transposed A
constexpr int TURN_BYTES = 32 * 16 * 4;                    // of a warp that empties tensor memory
constexpr int RASTER_ROWS = 2048;                          // rows of row tiles that share a pass over the columns

struct alignas(64) GemmArgs {
  CUtensorMap a[3], b[3];                                  // (GLU: b[2] and a[1] are Wg and Wu in boxes of 32 rows)
  int4* plan;                                              // {tiles, ok, the first products failed, -}, then {first row, rows, expert, -} of every tile
  const int32_t* offsets;
  int R, D, I, E, groups;
  void* out[3];
  const float* in[2];                                      // a and u of the forward pass
  float* keep[2];                                          // and where it leaves them, or NULL
  int32_t* status;
};

// ---- PTX ------------------------------------------------------------------------------------------------

__device__ __forceinline__ void barrier_init(unsigned bar, unsigned count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_expect(unsigned bar, unsigned bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void barrier_arrive(unsigned bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// whether the phase is over: a look that does not wait
__device__ __forceinline__ unsigned barrier_passed(unsigned bar, unsigned parity) {
  unsigned done;
  asm volatile("{\n.reg .pred p;\nmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
               : "=r"(done) : "r"(bar), "r"(parity) : "memory");
  return done;
}
// Waits for the phase, but not for ever: false if it gave up, or if somebody else of the CTA has (a bug, never an input). The look
// comes first because a wait takes 200 cycles even where there is nothing to wait for, and the look 100.
__device__ __forceinline__ bool barrier_wait(unsigned bar, unsigned parity, volatile int* failed, int most) {
  if (barrier_passed(bar, parity)) return true;
  for (int tries = 0; tries < most; ++tries) {
    unsigned done;                                         // (waits for a microsecond at most)
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\nselp.u32 %0, 1, 0, p;\n}"
                 : "=r"(done) : "r"(bar), "r"(parity), "r"(1000u) : "memory");
    if (done) return true;
    if ((tries & 255) == 255 && *failed) return false;
  }
  *failed = 1;
  return false;
}
// For a whole warp: what follows is the same for all lanes, and the compiler sees it. (The descriptors of matrix instructions and
// copies are read from the warp's common registers; out of a branch of one lane they were moved there one by one, which
// took 80 to 130 cycles an instruction and was what bounded the products.)
__device__ __forceinline__ bool warp_wait(unsigned bar, unsigned parity, volatile int* failed, int most) {
  return __all_sync(FULL, barrier_wait(bar, parity, failed, most)) != 0;
}
__device__ __forceinline__ bool elect_lane() {
  unsigned is;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(is));
  return is != 0;
}
// the address of `local` in CTA `rank` of the cluster
__device__ __forceinline__ unsigned in_cta(unsigned local, unsigned rank) {
  unsigned out;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(out) : "r"(local), "r"(rank));
  return out;
}
__device__ __forceinline__ void barrier_arrive_in(unsigned remote) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(remote) : "memory");
}
__device__ __forceinline__ void tma_load(unsigned dst, const CUtensorMap* map, unsigned bar, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
// into this CTA, counted on a barrier that may be the other CTA's of the pair
__device__ __forceinline__ void tma_load_pair(unsigned dst, const CUtensorMap* map, unsigned bar, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void mma_issue(unsigned d, unsigned long long a, unsigned long long b, unsigned idesc, bool add) {
  if constexpr (PAIR)
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((unsigned)add) : "memory");
  else
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((unsigned)add) : "memory");
}
// an arrival at the barrier (of a pair: of both CTAs) when the matrix instructions issued so far are done
template <bool PAIR>
__device__ __forceinline__ void mma_commit(unsigned bar) {
  if constexpr (PAIR)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((unsigned short)3) : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// Loads from tensor memory are instructions of a whole warp (.aligned): where lanes may have gone different ways before, as at the
// ragged ends of rows and columns, __syncwarp() brings them together first.
__device__ __forceinline__ void tmem_load16(unsigned addr, float (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]),
        "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_load32(unsigned addr, float (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]),
        "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]),
        "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]),
        "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Operand in shared memory, swizzled by 128 bytes. Contraction along the rows of 128 bytes: groups of 8 rows are 1024 bytes apart.
// Transposed (a row of 128 bytes holds 64 rows or columns of the result at one k): 8 k are 1024 bytes, the next 64 rows or
// columns of the result one box further on.
__device__ __forceinline__ unsigned long long operand(unsigned addr, bool transposed) {
  const unsigned long long lead = transposed ? BOX_BYTES >> 4 : 1;
  return (unsigned long long)((addr >> 4) & 0x3fff) | lead << 16 | (1024ull >> 4) << 32 | 1ull << 46 | 2ull << 61;
}

// ---- row tiles ------------------------------------------------------------------------------------------

// Tiles of up to `high` rows of the groups, by expert, so that tiles with the same weights follow one another. One CTA, of a thread
// for each group up to 1024.
__global__ void __launch_bounds__(1024) plan_kernel(int R, int E, int groups, int high, const int32_t* __restrict__ offsets,
                                                    int4* __restrict__ plan, int32_t* __restrict__ status) {
  __shared__ int warp_sum[32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, threads = blockDim.x, per = groups / E;
  let_next_start();
  bool bad = false;
  for (int g = threadIdx.x; g < groups; g += threads) {
    const int v = offsets[g], w = offsets[g + 1];
    bad |= v < 0 || v > w || w > R;
  }
  bad = __syncthreads_or(bad);
  int base = 0;
  for (int q0 = 0; q0 < groups && !bad; q0 += threads) {
    const int q = q0 + threadIdx.x, e = q / per;
    const int2 span = q < groups ? rows_of_group(offsets, (q - e * per) * E + e, R) : make_int2(0, 0);
    const int tiles = (span.y - span.x + high - 1) / high;
    int incl = tiles;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(FULL, incl, o);
      if (lane >= o) incl += v;
    }
    if (lane == 31) warp_sum[warp] = incl;
    __syncthreads();
    int before = base, all = base;
    for (int w = 0; w < threads / 32; ++w) {
      before += w < warp ? warp_sum[w] : 0;
      all += warp_sum[w];
    }
    for (int i = 0; i < tiles; ++i)
      plan[1 + before + incl - tiles + i] = make_int4(span.x + i * high, min(high, span.y - span.x - i * high), e, 0);
    base = all;
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    plan[0] = make_int4(bad ? 0 : base, !bad, 0, 0);
    *status = bad ? MOESCHED_ST_BAD_INPUT : MOESCHED_ST_OK;
  }
}

// Gradients of the weights where there are no rows: 0, or NaN where the offsets name some.
__global__ void __launch_bounds__(1024) no_rows_kernel(const int4* plan, void* dw_gate, void* dw_up, void* dw_down, size_t bytes) {
  const unsigned value = plan[0].y ? 0 : NANS;
  fill(dw_gate, bytes, value, blockIdx.x, gridDim.x);
  fill(dw_up, bytes, value, blockIdx.x, gridDim.x);
  fill(dw_down, bytes, value, blockIdx.x, gridDim.x);
}

// ---- the products ---------------------------------------------------------------------------------------

struct Tile {
  int row, rows, e, n;      // first row of the result and rows, expert, first column
  int which;                // DWEIGHT: 0 gate, 1 up, 2 down
  bool narrow;              // half of a tile's columns
};
// a tile of MODE is M rows high and N columns wide; GLU's are made of as many products again
template <int MODE, bool PAIR>
struct Shape {
  static constexpr int M = PAIR ? 2 * CTA_M : CTA_M, SUMS = PAIR ? 2 * CTA_N : CTA_N, N = MODE == GLU ? SUMS / 2 : SUMS;
};
__host__ __device__ constexpr long long div_up(long long a, long long b) { return (a + b - 1) / b; }

template <int MODE, bool PAIR>
__device__ __forceinline__ int tile_total(const GemmArgs& a, const int4 head) {
  using S = Shape<MODE, PAIR>;
  if constexpr (MODE == DWEIGHT) {
    const int gu = (int)(div_up(a.I, S::M) * div_up(a.D, S::N)), dn = (int)(div_up(a.D, S::M) * div_up(a.I, S::N));
    return a.E * (2 * gu + dn);
  } else {
    return head.x * (int)div_up(MODE == GLU || MODE == DHIDDEN ? a.I : a.D, S::N);
  }
}
// Of `total` tiles for `step` CTAs or pairs, those of a last, or only, round that at most half of them would have are cut in two:
// tiles up to `whole` are whole, the others come as halves. (DWEIGHT's tiles have short contractions, or many rounds.)
template <int MODE, bool PAIR>
__device__ __forceinline__ int whole_tiles(int total, int step) {
  const int last = total % step;
  return MODE != DWEIGHT && 2 * last <= step ? total - last : total;
}
template <int MODE, bool PAIR>
__device__ __forceinline__ Tile tile_at(const GemmArgs& a, const int4 head, int t, int whole) {
  using S = Shape<MODE, PAIR>;
  Tile w;
  w.narrow = t >= whole;
  const int second = w.narrow ? (t - whole) & 1 : 0;
  if (w.narrow) t = whole + (t - whole) / 2;
  if constexpr (MODE == DWEIGHT) {
    const int gu = (int)(div_up(a.I, S::M) * div_up(a.D, S::N)), dn = (int)(div_up(a.D, S::M) * div_up(a.I, S::N));
    const int each = 2 * gu + dn;
    w.e = t / each;
    t -= w.e * each;
    w.which = t < gu ? 0 : t < 2 * gu ? 1 : 2;
    t -= w.which * gu;
    const int M = w.which < 2 ? a.I : a.D, m_tiles = (int)div_up(M, S::M);
    w.row = t % m_tiles * S::M;
    w.rows = min(S::M, M - w.row);
    w.n = t / m_tiles * S::N;
  } else {
    constexpr int RASTER = RASTER_ROWS / S::M;
    const int n_tiles = (int)div_up(MODE == GLU || MODE == DHIDDEN ? a.I : a.D, S::N);
    const int block = t / (RASTER * n_tiles), first = block * RASTER, high = min(RASTER, head.x - first);
    t -= first * n_tiles;
    const int4 row = a.plan[1 + first + t % high];
    w.row = row.x, w.rows = row.y, w.e = row.z, w.n = t / high * S::N + second * (S::N / 2), w.which = 0;
  }
  return w;
}
// The groups of an expert, for DWEIGHT: the first one's rows are kept from tile to tile, the next one's are on their way while
// one is worked on.
struct Spans {
  int expert = -1, begin = 0, end = 0;
};
// NaN in all outputs of a product (hidden rows and their gradients are nobody's)
template <int MODE>
__device__ __forceinline__ void spoil(const GemmArgs& a, unsigned part, unsigned parts) {
  if constexpr (MODE == GLU) {
    for (int q = 0; q < 2 && a.keep[0] != nullptr; ++q) fill(a.keep[q], (size_t)a.R * a.I * 4, NANS, part, parts);
  } else if constexpr (MODE == DWEIGHT) {
    for (int q = 0; q < 3; ++q) fill(a.out[q], (size_t)a.E * a.I * a.D * 2, NANS, part, parts);
  } else if constexpr (MODE != DHIDDEN) {
    fill(a.out[0], (size_t)a.R * a.D * 2, NANS, part, parts);
  }
}

// calls f(k-block's first row or column, what it holds (64 or less), which operands) for every block of the contraction
template <int MODE, typename F>
__device__ __forceinline__ bool each_block(const GemmArgs& a, const Tile& w, Spans& kept, F&& f) {
  if constexpr (MODE == DWEIGHT) {
    if (kept.expert != w.e) kept = {w.e, a.offsets[w.e], a.offsets[w.e + 1]};
    int begin = kept.begin, end = kept.end;
    for (int g = w.e; g < a.groups; g += a.E) {
      const bool more = g + a.E < a.groups;
      const int next_begin = more ? a.offsets[g + a.E] : 0, next_end = more ? a.offsets[g + a.E + 1] : 0;
      for (int r = begin; r < end; r += BK)                // (the plan has found all offsets in order)
        if (!f(r, min(BK, end - r), w.which)) return false;
      begin = next_begin, end = next_end;
    }
  } else {
    const int K = MODE == GLU || MODE == DHIDDEN ? a.D : a.I;
    for (int part = 0; part < (MODE == DINPUT ? 2 : 1); ++part)
      for (int k = 0; k < K; k += BK)
        if (!f(k, BK, part)) return false;
  }
  return true;
}

// place of the four words `part` of row `row` in a warp's 32 x 16 words: rows that lanes store and rows that they load together
// lie in different banks
__device__ __forceinline__ float4* turned(float* base, int row, int part) {
  return reinterpret_cast<float4*>(base + row * 16 + ((part ^ (row >> 1 & 3)) << 2));
}

template <int MODE, bool PAIR, typename T, int ACT>
__global__ void __launch_bounds__(GEMM_THREADS, 1) gemm_kernel(const __grid_constant__ GemmArgs a) {
  using S = Shape<MODE, PAIR>;
  constexpr bool A_T = MODE == DWEIGHT, B_T = MODE == DHIDDEN || MODE == DINPUT || MODE == DWEIGHT;
  constexpr int TMEM_COLUMNS = 2 * S::SUMS;
  extern __shared__ unsigned char raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  unsigned long long* bars = reinterpret_cast<unsigned long long*>(smem + STAGES * STAGE_BYTES + EMPTIERS * TURN_BYTES);
  const unsigned ring = smem_addr(smem);
  // full, done: operands there, sums there; empty, free_: may be overwritten; partly, fixed: blocks that end within (DWEIGHT)
  const unsigned full = smem_addr(bars), empty = full + 8 * STAGES, partly = empty + 8 * STAGES, fixed = partly + 8 * STAGES,
                 done = fixed + 8 * STAGES, free_ = done + 16, drain = free_ + 16;
  int* words = reinterpret_cast<int*>(bars + 4 * STAGES + 5);
  volatile int* failed = words;
  // Looks at a barrier before a wait gives up: seconds. DWEIGHT's contractions are as long as an expert has rows and groups.
  const int patience = (1 << 22) + (MODE == DWEIGHT ? 32 * (a.R / BK + a.groups) : 0);
  const int lane = threadIdx.x & 31, warp = __shfl_sync(FULL, (int)threadIdx.x >> 5, 0);
  const unsigned rank = PAIR ? cluster_ctarank() : 0;      // the first CTA of a pair issues
  const int first_tile = PAIR ? blockIdx.x / 2 : blockIdx.x, step = PAIR ? gridDim.x / 2 : gridDim.x;
  Spans spans;
  let_next_start();

  if (threadIdx.x == 0) {
    *failed = 0;
    for (int s = 0; s < STAGES; ++s) {
      barrier_init(full + 8 * s, 1);
      barrier_init(empty + 8 * s, 1);
      barrier_init(partly + 8 * s, 1);
      barrier_init(fixed + 8 * s, PAIR ? 2 : 1);
    }
    for (int q = 0; q < 2; ++q) {
      barrier_init(done + 8 * q, 1);
      barrier_init(free_ + 8 * q, (PAIR ? 2 : 1) * EMPTIERS);
    }
    barrier_init(drain, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    if constexpr (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(words + 1)), "n"(TMEM_COLUMNS) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(words + 1)), "n"(TMEM_COLUMNS) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  fence_before();
  __syncthreads();
  if constexpr (PAIR) cluster_sync_all();                  // the other CTA's barriers are there
  fence_after();
  const unsigned tmem = *reinterpret_cast<volatile unsigned*>(words + 1);
  wait_for_previous();                                     // nothing of other kernels is read, and nothing written, before
  const int4 head = a.plan[0];
  // (head.z, that GLU or DHIDDEN gave up, is the same for all CTAs of the products that follow; those two do not look at it)
  constexpr bool FIRST = MODE == GLU || MODE == DHIDDEN;
  const bool lost = !head.y || (!FIRST && head.z);
  if (lost) spoil<MODE>(a, blockIdx.x, gridDim.x);
  const int tiles = lost ? 0 : tile_total<MODE, PAIR>(a, head), whole = whole_tiles<MODE, PAIR>(tiles, step), total = 2 * tiles - whole;

  if (warp == 0) {
    const bool elected = elect_lane();
    int stage = 0, issued = 0;
    unsigned phase = 0;
    bool ok = true;
    const unsigned lead_full = PAIR ? in_cta(full, 0) : full;
    Tile next = first_tile < total ? tile_at<MODE, PAIR>(a, head, first_tile, whole) : Tile{};
    for (int t = first_tile; t < total && ok; t += step) {
      const Tile w = next;
      const int row = w.row + (int)rank * CTA_M, begun = issued;
      bool looked = false;                               // where the next tile is, while there is a wait anyway
      const auto look_ahead = [&]() {
        looked = true;
        if (t + step < total) next = tile_at<MODE, PAIR>(a, head, t + step, whole);
      };
      ok = each_block<MODE>(a, w, spans, [&](int k, int held, int part) {
        if (issued == begun + 3) look_ahead();
        if (!warp_wait(empty + 8 * stage, phase ^ 1, failed, patience)) return false;
        const unsigned to = ring + stage * STAGE_BYTES, tb = to + A_BYTES;
        // a block that ends within is counted by each CTA for itself, for the warp that zeroes its end
        const bool own = MODE == DWEIGHT && held < BK;
        const unsigned bar = own ? partly + 8 * stage : lead_full + 8 * stage;
        if (elected) {
          if (own) barrier_expect(bar, STAGE_BYTES);
          else if (rank == 0) barrier_expect(full + 8 * stage, (PAIR ? 2 : 1) * (w.narrow ? STAGE_BYTES - B_BYTES / 2 : STAGE_BYTES));
          const auto load = [&](unsigned dst, const CUtensorMap* map, int x, int y, int z) {
            if (PAIR && !own) tma_load_pair(dst, map, bar, x, y, z);
            else tma_load(dst, map, bar, x, y, z);
          };
          if constexpr (A_T) {
            for (int q = 0; q < 2; ++q) load(to + q * BOX_BYTES, &a.a[part], row + 64 * q, k, 0);
          } else {
            load(to, &a.a[MODE == DINPUT ? part : 0], k, row, 0);
          }
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            if (q == 1 && w.narrow) break;
            const unsigned dst = tb + q * BOX_BYTES;
            if constexpr (MODE == GLU) {                   // a pair: a of the first CTA, u of the second
              if constexpr (PAIR) {
                load(dst, &a.b[rank], k, w.n + 64 * q, w.e);
              } else if (w.narrow) {
                load(tb, &a.b[2], k, w.n, w.e);
                load(tb + BOX_BYTES / 2, &a.a[1], k, w.n, w.e);
              } else {
                load(dst, &a.b[q], k, w.n, w.e);
              }
            } else {
              const int n = w.n + (int)rank * (w.narrow ? CTA_N / 2 : CTA_N) + 64 * q;
              if constexpr (MODE == DOWN) load(dst, &a.b[0], k, n, w.e);
              else load(dst, &a.b[MODE == DHIDDEN ? 0 : part], n, k, MODE == DWEIGHT ? 0 : w.e);
            }
          }
        }
        ++issued;
        if (++stage == STAGES) stage = 0, phase ^= 1;
        return true;
      });
      if (!looked) look_ahead();
    }
    if (!ok) {                                            // nothing may land in shared memory that is no longer ours
      const long long now = clock64();
      while (clock64() - now < 10'000'000) __nanosleep(1000);
    }
  } else if (warp == 1) {
    if (rank == 0) {
      const bool elected = elect_lane();
      constexpr unsigned FORMAT = std::is_same_v<T, __half> ? 0 : 1;
      constexpr unsigned IDESC = 1u << 4 | FORMAT << 7 | FORMAT << 10 | (A_T ? 1u : 0u) << 15 | (B_T ? 1u : 0u) << 16 |
                                 (S::SUMS / 8) << 17 | (S::M / 16) << 24, NARROW = IDESC - ((S::SUMS / 16) << 17);
      int stage = 0, slot = 0;
      unsigned phase = 0, slot_phase = 0, fixed_phase = 0, full_phase = 0;
      bool ok = true, ready = false;                       // ready: the next block's operands have been seen there
      for (int t = first_tile; t < total && ok; t += step) {
        const Tile w = tile_at<MODE, PAIR>(a, head, t, whole);
        bool first = true;
        const unsigned d = tmem + slot * S::SUMS, idesc = w.narrow ? NARROW : IDESC;
        ok = each_block<MODE>(a, w, spans, [&](int, int held, int) {
          if (first && !warp_wait(free_ + 8 * slot, slot_phase ^ 1, failed, patience)) return false;
          const bool partial = MODE == DWEIGHT && held < BK;
          if (partial) {
            if (!warp_wait(fixed + 8 * stage, fixed_phase >> stage & 1, failed, patience)) return false;
            fixed_phase ^= 1u << stage;
          } else {                                          // (blocks that end within pass `full` by)
            if (!ready && !warp_wait(full + 8 * stage, MODE == DWEIGHT ? full_phase >> stage & 1 : phase, failed, patience)) return false;
            full_phase ^= 1u << stage;
          }
          fence_after();
          // the look at the next block's operands takes its 100 cycles while this block's products are issued, which with the
          // waits is all that bounds a CTA's only tile (DWEIGHT's next block may be another warp's to finish first)
          const int then = stage + 1 == STAGES ? 0 : stage + 1;
          const unsigned seen = MODE == DWEIGHT ? 0 : barrier_passed(full + 8 * then, then ? phase : phase ^ 1);
          const unsigned at = ring + stage * STAGE_BYTES;
          const unsigned long long da = operand(at, A_T), db = operand(at + A_BYTES, B_T);
          // 16 k: 32 bytes of a row, or 16 rows of 128 bytes
          constexpr int A_STEP = A_T ? 2048 >> 4 : 32 >> 4, B_STEP = B_T ? 2048 >> 4 : 32 >> 4;
          if (elected) {
            mma_issue<PAIR>(d, da, db, idesc, !first);
            if (!partial) {
#pragma unroll
              for (int s = 1; s < BK / 16; ++s) mma_issue<PAIR>(d, da + s * A_STEP, db + s * B_STEP, idesc, true);
            } else {
              for (int s = 1; s < (held + 15) / 16; ++s) mma_issue<PAIR>(d, da + s * A_STEP, db + s * B_STEP, idesc, true);
            }
            mma_commit<PAIR>(empty + 8 * stage);
          }
          __syncwarp();
          ready = __all_sync(FULL, seen);
          first = false;
          if (++stage == STAGES) stage = 0, phase ^= 1;
          return true;
        });
        if (!first) {
          if (elected) mma_commit<PAIR>(done + 8 * slot);
          if (++slot == 2) slot = 0, slot_phase ^= 1;
        }
      }
      if (!ok) {
        if (elected) mma_commit<PAIR>(drain);
        int never = 0;
        barrier_wait(drain, 0, &never, 1 << 22);
      }
    }
  } else if (warp == 2) {
    if constexpr (MODE == DWEIGHT) {                        // zeroes what a block holds behind its group's last row
      int stage = 0;
      unsigned part_phase = 0;
      bool ok = true;
      const unsigned lead_fixed = PAIR ? in_cta(fixed, 0) : fixed;
      for (int t = first_tile; t < total && ok; t += step) {
        const Tile w = tile_at<MODE, PAIR>(a, head, t, whole);
        ok = each_block<MODE>(a, w, spans, [&](int, int held, int) {
          if (held < BK) {
            if (!__all_sync(FULL, barrier_wait(partly + 8 * stage, part_phase >> stage & 1, failed, patience))) return false;
            part_phase ^= 1u << stage;
            const int to = (held + 15) / 16 * 16, bytes16 = (to - held) * 8;
            unsigned char* from = smem + stage * STAGE_BYTES + held * 128;
            for (int at = lane; at < bytes16; at += 32)
#pragma unroll
              for (int box = 0; box < 4; ++box) *reinterpret_cast<uint4*>(from + box * BOX_BYTES + at * 16) = make_uint4(0, 0, 0, 0);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
              if constexpr (PAIR) barrier_arrive_in(lead_fixed + 8 * stage);
              else barrier_arrive(fixed + 8 * stage);
            }
          }
          if (++stage == STAGES) stage = 0;
          return true;
        });
      }
    }
  } else if (warp >= 4) {
    const int quarter = warp & 3, half = (warp - 4) >> 2;  // lanes of tensor memory, and which half of the columns
    const unsigned mine = tmem + ((unsigned)quarter << 21);
    const unsigned lead_free = PAIR ? in_cta(free_, 0) : free_;
    float* turn = reinterpret_cast<float*>(smem + STAGES * STAGE_BYTES + (warp - 4) * TURN_BYTES);
    // after the turn a lane has, in round q, four words of row 8 q + lane / 4
    const int t_row = lane >> 2, t_part = lane & 3;
    int slot = 0;
    unsigned slot_phase = 0;
    for (int t = first_tile; t < total; t += step) {
      const Tile w = tile_at<MODE, PAIR>(a, head, t, whole);
      const int row = w.row + (int)rank * CTA_M + quarter * 32 + t_row;       // of round 0
      const int rows = w.rows - ((int)rank * CTA_M + quarter * 32 + t_row);  // round q is inside if 8 q < rows
      const unsigned d = mine + slot * S::SUMS;
      const int columns = w.narrow ? S::N / 2 : S::N, c_begin = half * (columns / 2), c_end = c_begin + columns / 2;
      bool any = true;
      if constexpr (MODE == DWEIGHT) {
        any = false;
        each_block<MODE>(a, w, spans, [&](int, int, int) { any = true; return false; });
      }
      const auto wait_sums = [&]() {
        if (!__all_sync(FULL, barrier_wait(done + 8 * slot, slot_phase, failed, patience))) return false;
        fence_after();
        return true;
      };
      if constexpr (MODE == GLU) {
        if (!wait_sums()) break;
        const size_t at = (size_t)row * a.I + w.n + 4 * t_part;
#pragma unroll 1
        for (int c = c_begin; c < c_end; c += 16) {
          float p[16], q[16];
          float4 gate[4];
          __syncwarp();                                    // (see tmem_load16)
          tmem_load16(d + c, p);
          tmem_load16(d + columns + c, q);
          tmem_load_wait();
          __syncwarp();
#pragma unroll
          for (int v = 0; v < 4; ++v) *turned(turn, lane, v) = make_float4(p[4 * v], p[4 * v + 1], p[4 * v + 2], p[4 * v + 3]);
          __syncwarp();
#pragma unroll
          for (int v = 0; v < 4; ++v) gate[v] = *turned(turn, 8 * v + t_row, t_part);
          __syncwarp();
#pragma unroll
          for (int v = 0; v < 4; ++v) *turned(turn, lane, v) = make_float4(q[4 * v], q[4 * v + 1], q[4 * v + 2], q[4 * v + 3]);
          __syncwarp();
          if (w.n + c + 4 * t_part < a.I) {
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              if (8 * v >= rows) continue;
              const float4 g = gate[v], u = *turned(turn, 8 * v + t_row, t_part);
              const size_t to = at + (size_t)(8 * v) * a.I + c;
              *reinterpret_cast<uint2*>(static_cast<T*>(a.out[0]) + to) =
                  make_uint2(Pair<T>::from_float(activation<ACT>(g.x) * u.x, activation<ACT>(g.y) * u.y),
                             Pair<T>::from_float(activation<ACT>(g.z) * u.z, activation<ACT>(g.w) * u.w));
              if (a.keep[0] != nullptr) {
                *reinterpret_cast<float4*>(a.keep[0] + to) = g;
                *reinterpret_cast<float4*>(a.keep[1] + to) = u;
              }
            }
          }
        }
      } else if constexpr (MODE == DHIDDEN) {
        const size_t at = (size_t)row * a.I + w.n + 4 * t_part;
        struct Held {
          float4 g[4], u[4];
        };
        const auto fetch = [&](int c, Held& h) {           // a and u of 16 columns, on their way while others are worked on
          const bool in = c < c_end && w.n + c + 4 * t_part < a.I;
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const size_t from = at + (size_t)(8 * v) * a.I + c;
            h.g[v] = h.u[v] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (in && 8 * v < rows) {
              h.g[v] = __ldcs(reinterpret_cast<const float4*>(a.in[0] + from));
              h.u[v] = __ldcs(reinterpret_cast<const float4*>(a.in[1] + from));
            }
          }
        };
        const auto work = [&](int c, const Held& h) {
          float p[16];
          __syncwarp();                                    // (see tmem_load16)
          tmem_load16(d + c, p);
          tmem_load_wait();
          __syncwarp();
#pragma unroll
          for (int v = 0; v < 4; ++v) *turned(turn, lane, v) = make_float4(p[4 * v], p[4 * v + 1], p[4 * v + 2], p[4 * v + 3]);
          __syncwarp();
          if (w.n + c + 4 * t_part >= a.I) return;
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            if (8 * v >= rows) continue;
            const float4 x = *turned(turn, 8 * v + t_row, t_part);
            const float xs[4] = {x.x, x.y, x.z, x.w}, gs[4] = {h.g[v].x, h.g[v].y, h.g[v].z, h.g[v].w},
                        us[4] = {h.u[v].x, h.u[v].y, h.u[v].z, h.u[v].w};
            float hid[4], dg[4], du[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float f, s;
              activation_slope<ACT>(gs[i], f, s);
              hid[i] = f * us[i], dg[i] = xs[i] * us[i] * s, du[i] = xs[i] * f;
            }
            const size_t to = at + (size_t)(8 * v) * a.I + c;
            *reinterpret_cast<uint2*>(static_cast<T*>(a.out[0]) + to) = make_uint2(Pair<T>::from_float(hid[0], hid[1]), Pair<T>::from_float(hid[2], hid[3]));
            *reinterpret_cast<uint2*>(static_cast<T*>(a.out[1]) + to) = make_uint2(Pair<T>::from_float(dg[0], dg[1]), Pair<T>::from_float(dg[2], dg[3]));
            *reinterpret_cast<uint2*>(static_cast<T*>(a.out[2]) + to) = make_uint2(Pair<T>::from_float(du[0], du[1]), Pair<T>::from_float(du[2], du[3]));
          }
        };
        Held even, odd;
        fetch(c_begin, even);
        fetch(c_begin + 16, odd);
        if (!wait_sums()) break;
#pragma unroll 1
        for (int c = c_begin; c < c_end; c += 32) {
          work(c, even);
          fetch(c + 32, even);
          work(c + 16, odd);
          fetch(c + 48, odd);
        }
      } else {
        if (any && !wait_sums()) break;
        const int cols = MODE == DWEIGHT && w.which == 2 ? a.I : a.D;
        const size_t first = MODE == DWEIGHT ? (size_t)w.e * a.I * a.D + (size_t)row * cols : (size_t)row * cols;
        T* out = static_cast<T*>(a.out[MODE == DWEIGHT ? w.which : 0]) + first + w.n + 8 * t_part;
#pragma unroll 1
        for (int c = c_begin; c < c_end; c += 32) {
          if (any) {
            float p[32];
            __syncwarp();                                  // (see tmem_load16)
            tmem_load32(d + c, p);
            tmem_load_wait();
            __syncwarp();
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              float4 words4;
              words4.x = __uint_as_float(Pair<T>::from_float(p[8 * v], p[8 * v + 1]));
              words4.y = __uint_as_float(Pair<T>::from_float(p[8 * v + 2], p[8 * v + 3]));
              words4.z = __uint_as_float(Pair<T>::from_float(p[8 * v + 4], p[8 * v + 5]));
              words4.w = __uint_as_float(Pair<T>::from_float(p[8 * v + 6], p[8 * v + 7]));
              *turned(turn, lane, v) = words4;
            }
            __syncwarp();
          }
          if (w.n + c + 8 * t_part < cols) {
#pragma unroll
            for (int v = 0; v < 4; ++v)
              if (8 * v < rows)
                *reinterpret_cast<float4*>(out + (size_t)(8 * v) * cols + c) =
                    any ? *turned(turn, 8 * v + t_row, t_part) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          }
        }
      }
      if (any) {
        fence_before();
        __syncwarp();
        if (lane == 0) {
          if constexpr (PAIR) barrier_arrive_in(lead_free + 8 * slot);
          else barrier_arrive(free_ + 8 * slot);
        }
        if (++slot == 2) slot = 0, slot_phase ^= 1;
      }
    }
  }
  fence_before();
  __syncthreads();
  if (*failed) {                                           // (what other CTAs still write does not reach this one's tiles)
    if (threadIdx.x == 0) {
      *a.status = MOESCHED_ST_INTERNAL;
      if (FIRST) a.plan[0].z = 1;
    }
    spoil<MODE>(a, 0, 1);
  }
  __syncwarp();
  if constexpr (PAIR) cluster_sync_all();                  // the other CTA may still use our barriers and operands
  if (warp == 1) {
    fence_after();
    if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(TMEM_COLUMNS));
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(TMEM_COLUMNS));
  }
}

// ---- host -----------------------------------------------------------------------------------------------

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static cudaError_t encoder(EncodeFn* fn) {
  static std::atomic<EncodeFn> kept{nullptr};              // (every thread finds the same)
  EncodeFn found = kept.load(std::memory_order_relaxed);
  if (found == nullptr) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult how;
    cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &how);
    if (e != cudaSuccess) return e;
    if (how != cudaDriverEntryPointSuccess || p == nullptr) return cudaErrorNotSupported;
    found = reinterpret_cast<EncodeFn>(p);
    kept.store(found, std::memory_order_relaxed);
  }
  *fn = found;
  return cudaSuccess;
}

// [deep][rows][cols] of a 16-bit type, in boxes of 64 columns and `high` rows
static cudaError_t make_map(EncodeFn encode, CUtensorMap* map, int dtype, const void* p, int cols, int rows, int deep, int high) {
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)deep};
  const cuuint64_t strides[2] = {(cuuint64_t)cols * 2, (cuuint64_t)cols * rows * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)high, 1}, step[3] = {1, 1, 1};
  const CUresult r = encode(map, dtype == MOESCHED_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3,
                            const_cast<void*>(p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

ExpertScratch expert_scratch(int R, int I, int groups, bool backward) {
  ExpertScratch s;
  size_t at = 0;
  const size_t table = ((size_t)R / CTA_M + groups + 1) * sizeof(int4), rows = (size_t)R * I * 2;
  auto take = [&](size_t bytes) {
    const size_t first = at;
    at += (bytes + 255) / 256 * 256;
    return first;
  };
  s.plan = take(table);
  s.hidden = take(rows);
  s.d_gate = backward ? take(rows) : 0;
  s.d_up = backward ? take(rows) : 0;
  s.bytes = at;
  return s;
}

template <int MODE, bool PAIR, typename T>
static cudaError_t launch_gemm(const GemmArgs& args, int act, cudaStream_t stream) {
  using S = Shape<MODE, PAIR>;
  auto kern = gemm_kernel<MODE, PAIR, T, MOESCHED_ACT_SILU>;
  if constexpr (MODE == GLU || MODE == DHIDDEN)            // (the others have no activation)
    if (act == MOESCHED_ACT_GELU) kern = gemm_kernel<MODE, PAIR, T, MOESCHED_ACT_GELU>;
  const size_t smem = 1024 + STAGES * STAGE_BYTES + EMPTIERS * TURN_BYTES + 8 * (4 * STAGES + 5) + 16;
  static_assert(1024 + STAGES * STAGE_BYTES + EMPTIERS * TURN_BYTES + 8 * (4 * STAGES + 5) + 16 <= SMEM_LIMIT, "shared memory");
  if (cudaError_t e = permit_shared_memory(kern, smem); e != cudaSuccess) return e;
  long long tiles;                                         // at most
  if (MODE == DWEIGHT)
    tiles = args.E * (2 * div_up(args.I, S::M) * div_up(args.D, S::N) + div_up(args.D, S::M) * div_up(args.I, S::N));
  else
    tiles = ((long long)args.R / S::M + (args.groups < args.R ? args.groups : args.R)) * div_up(MODE == GLU || MODE == DHIDDEN ? args.I : args.D, S::N);
  const long long most = PAIR ? sm_count() / 2 : sm_count();
  cudaLaunchConfig_t cfg = {};
  const long long units = MODE == DWEIGHT ? tiles : 2 * tiles;   // (halves)
  cfg.gridDim = dim3((unsigned)((units < most ? units : most) * (PAIR ? 2 : 1)));
  cfg.blockDim = dim3(GEMM_THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0] = start_early();
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 2;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = PAIR ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, args);
}
template <int MODE>
static cudaError_t launch_gemm(const GemmArgs& args, bool pair, int dtype, int act, cudaStream_t stream) {
  if (dtype == MOESCHED_BF16)
    return pair ? launch_gemm<MODE, true, __nv_bfloat16>(args, act, stream) : launch_gemm<MODE, false, __nv_bfloat16>(args, act, stream);
  return pair ? launch_gemm<MODE, true, __half>(args, act, stream) : launch_gemm<MODE, false, __half>(args, act, stream);
}

static int plan_threads(int groups) { return groups >= 1024 ? 1024 : (groups + 31) / 32 * 32; }

// A handful of rows for each expert: the kernel that streams the weights, once for every eight rows of an expert. (Four experts of
// 7168 x 2048: 25 us for one row and 68 for 24, row tiles 49 and 84; from nine rows an expert on it would read weights twice, 130
// us for 48 rows and 69. Rows may be spread unevenly, hence four, and eight more, which few experts can take.)
static bool few_rows(int R, int E) { return R <= 4LL * E + 8; }

// Tiles of pairs or of single CTAs? A pair does some 1.4 times as much as its two SMs would alone, but its tiles are four times
// as large. Single CTAs where their tiles of every product find an SM each (one expert, 4096 x 2048, 330 rows: 37 us, pairs 44;
// 700 rows, two rounds: 64 and 47), or where groups have less than 128 rows on the average, more than half of a tile of 256
// rows then being empty. (Each group is taken to fill half of its last tile.)
static bool tiles_of_pairs(int R, int D, int I, int groups) {
  if (R / CTA_M < groups) return false;
  const long long high = div_up(R + (long long)groups * (CTA_M / 2), CTA_M);
  return high * div_up(I, CTA_N / 2) > sm_count() || high * div_up(D, CTA_N) > sm_count();
}

cudaError_t run_expert_ffn(int R, int D, int I, int E, int groups, int dtype, int act, const void* x, const void* w_gate,
                           const void* w_up, const void* w_down, const int32_t* offsets, void* y, float* gate, float* up,
                           void* scratch, int32_t* status, cudaStream_t stream) {
  const ExpertScratch at = expert_scratch(R, I, groups, false);
  unsigned char* base = static_cast<unsigned char*>(scratch);
  void* hidden = base + at.hidden;
  cudaError_t e;
  if (few_rows(R, E)) {
    e = run_few(R, D, I, E, groups, 0, dtype, act, x, w_gate, nullptr, w_up, nullptr, offsets, hidden, gate, up, status, false,
                stream);
    if (e != cudaSuccess) return e;
    return run_few(R, I, D, E, groups, 0, dtype, act, hidden, w_down, nullptr, nullptr, nullptr, offsets, y, nullptr, nullptr,
                   status, true, stream);
  }
  EncodeFn encode;
  if ((e = encoder(&encode)) != cudaSuccess) return e;
  const bool pair = tiles_of_pairs(R, D, I, groups);
  int4* plan = reinterpret_cast<int4*>(base + at.plan);
  GemmArgs args[2] = {};
  for (GemmArgs& g : args) {
    g.plan = plan;
    g.offsets = offsets;
    g.R = R, g.D = D, g.I = I, g.E = E, g.groups = groups;
    g.status = status;
  }
  const auto map = [&](CUtensorMap* m, const void* p, int cols, int rows, int deep, int high) {
    if (e == cudaSuccess) e = make_map(encode, m, dtype, p, cols, rows, deep, high);
  };
  map(&args[0].a[0], x, D, R, 1, CTA_M);
  map(&args[0].b[0], w_gate, D, I, E, 64);
  map(&args[0].b[1], w_up, D, I, E, 64);
  if (!pair) {
    map(&args[0].b[2], w_gate, D, I, E, 32);
    map(&args[0].a[1], w_up, D, I, E, 32);
  }
  args[0].out[0] = hidden, args[0].keep[0] = gate, args[0].keep[1] = up;
  map(&args[1].a[0], hidden, I, R, 1, CTA_M);
  map(&args[1].b[0], w_down, I, D, E, 64);
  args[1].out[0] = y;
  if (e != cudaSuccess) return e;
  plan_kernel<<<1, plan_threads(groups), 0, stream>>>(R, E, groups, pair ? 2 * CTA_M : CTA_M, offsets, plan, status);
  if ((e = cudaGetLastError()) != cudaSuccess) return e;
  if ((e = launch_gemm<GLU>(args[0], pair, dtype, act, stream)) != cudaSuccess) return e;
  return launch_gemm<DOWN>(args[1], pair, dtype, act, stream);
}

cudaError_t run_expert_backward(int R, int D, int I, int E, int groups, int dtype, int act, const void* dy, const void* x,
                                const void* w_gate, const void* w_up, const void* w_down, const int32_t* offsets,
                                const float* gate, const float* up, void* dx, void* dw_gate, void* dw_up, void* dw_down,
                                void* scratch, int32_t* status, cudaStream_t stream) {
  cudaError_t e;
  const size_t weights = (size_t)E * I * D * 2;
  const bool pair = tiles_of_pairs(R, D, I, groups);
  if (R == 0) {                                             // no rows: no tensor maps, and gradients of nothing
    int4* plan = static_cast<int4*>(scratch);
    plan_kernel<<<1, plan_threads(groups), 0, stream>>>(R, E, groups, CTA_M, offsets, plan, status);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    no_rows_kernel<<<sm_count(), 1024, 0, stream>>>(plan, dw_gate, dw_up, dw_down, weights);
    return cudaGetLastError();
  }
  const ExpertScratch at = expert_scratch(R, I, groups, true);
  unsigned char* base = static_cast<unsigned char*>(scratch);
  void *hidden = base + at.hidden, *d_gate = base + at.d_gate, *d_up = base + at.d_up;
  EncodeFn encode;
  if ((e = encoder(&encode)) != cudaSuccess) return e;
  int4* plan = reinterpret_cast<int4*>(base + at.plan);
  GemmArgs args[3] = {};
  for (GemmArgs& g : args) {
    g.plan = plan;
    g.offsets = offsets;
    g.R = R, g.D = D, g.I = I, g.E = E, g.groups = groups;
    g.status = status;
  }
  const auto map = [&](CUtensorMap* m, const void* p, int cols, int rows, int deep, int high) {
    if (e == cudaSuccess) e = make_map(encode, m, dtype, p, cols, rows, deep, high);
  };
  map(&args[0].a[0], dy, D, R, 1, CTA_M);
  map(&args[0].b[0], w_down, I, D, E, BK);
  args[0].in[0] = gate, args[0].in[1] = up;
  args[0].out[0] = hidden, args[0].out[1] = d_gate, args[0].out[2] = d_up;
  map(&args[1].a[0], d_gate, I, R, 1, CTA_M);
  map(&args[1].a[1], d_up, I, R, 1, CTA_M);
  map(&args[1].b[0], w_gate, D, I, E, BK);
  map(&args[1].b[1], w_up, D, I, E, BK);
  args[1].out[0] = dx;
  map(&args[2].a[0], d_gate, I, R, 1, BK);
  map(&args[2].a[1], d_up, I, R, 1, BK);
  map(&args[2].a[2], dy, D, R, 1, BK);
  map(&args[2].b[0], x, D, R, 1, BK);
  args[2].b[1] = args[2].b[0];
  map(&args[2].b[2], hidden, I, R, 1, BK);
  args[2].out[0] = dw_gate, args[2].out[1] = dw_up, args[2].out[2] = dw_down;
  if (e != cudaSuccess) return e;
  plan_kernel<<<1, plan_threads(groups), 0, stream>>>(R, E, groups, pair ? 2 * CTA_M : CTA_M, offsets, plan, status);
  if ((e = cudaGetLastError()) != cudaSuccess) return e;
  if ((e = launch_gemm<DHIDDEN>(args[0], pair, dtype, act, stream)) != cudaSuccess) return e;
  if ((e = launch_gemm<DINPUT>(args[1], pair, dtype, act, stream)) != cudaSuccess) return e;
  return launch_gemm<DWEIGHT>(args[2], pair, dtype, act, stream);
}

}  // namespace moesched
