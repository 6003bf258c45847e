// Gated feed-forward block of the experts on rows grouped by expert, and its backward pass: five products on the tensor
// cores, with what stands between them in their epilogues.
//
//   GLU      a = X Wg^T, u = X Wu^T                    -> h = act(a) u (and a, u for the backward pass)
//   DOWN     y = h Wd^T
//   DHIDDEN  dh = dY Wd                                -> h again, du = dh act(a), da = dh u act'(a)
//   DINPUT   dX = da Wg + du Wu                        (one contraction over 2 I)
//   DWEIGHT  dWg = da^T X, dWu = du^T X, dWd = dY^T h  (contractions over the rows of an expert)
//
// A persistent CTA per SM takes tiles of 128 x 256 (GLU: 128 columns of a and the same 128 of u). One warp fetches the operands with TMA,
// 64 deep, into a ring of stages; one thread issues the matrix instructions, whose sums are in tensor memory, twice, so that four
// warps empty one while the other fills. Operands stay as they are in memory: where the contraction runs over
// the slower axis (Wd in DHIDDEN, Wg and Wu in DINPUT, everything in DWEIGHT) the instruction takes them transposed.
// Row tiles of the groups are laid out by a small kernel first (plan_kernel): a tile never spans two groups, what lies behind its
// group's last row is computed and not stored. In DWEIGHT the rows are the contraction: there the rows behind
// a group's last, up to the next multiple of 16, are zeroed in shared memory (0 x NaN would not be nothing).
#include <cuda.h>

#include "expert.cuh"

namespace moesched {

enum { GLU, DOWN, DHIDDEN, DINPUT, DWEIGHT };

constexpr int BM = 128, BN = 256, BK = 64;
constexpr int STAGES = 4;
constexpr int A_BYTES = BM * BK * 2, B_BYTES = BN * BK * 2, STAGE_BYTES = A_BYTES + B_BYTES;
constexpr int GEMM_THREADS = 256;
constexpr int MAP_BOX_BYTES = 64 * 64 * 2;                 // one box of a transposed operand
constexpr int RASTER = 16;                                 // row tiles that share a pass over the columns

struct alignas(64) GemmArgs {
  CUtensorMap a[3], b[3];
  const int4* plan;                                        // {tiles, ok, -, -}, then {first row, rows, expert, -} of every tile
  const int32_t* offsets;
  int R, D, I, E, groups;
  void* out[3];
  const void* in[2];
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
// Waits for the phase, but not for ever: false if it gave up, or if somebody else of the CTA has (a bug, never an input).
__device__ __forceinline__ bool barrier_wait(unsigned bar, unsigned parity, volatile int* failed) {
  for (int tries = 0; tries < (1 << 22); ++tries) {
    unsigned done;                                         // (waits for a microsecond at most)
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\nselp.u32 %0, 1, 0, p;\n}"
                 : "=r"(done) : "r"(bar), "r"(parity), "r"(1000u) : "memory");
    if (done) return true;
    if ((tries & 255) == 255 && *failed) return false;
  }
  *failed = 1;
  return false;
}
__device__ __forceinline__ void tma_load(unsigned dst, const CUtensorMap* map, unsigned bar, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void mma_issue(unsigned d, unsigned long long a, unsigned long long b, unsigned idesc, bool add) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((unsigned)add) : "memory");
}
__device__ __forceinline__ void mma_commit(unsigned bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
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
  const unsigned long long lead = transposed ? MAP_BOX_BYTES >> 4 : 1;
  return (unsigned long long)((addr >> 4) & 0x3fff) | lead << 16 | (1024ull >> 4) << 32 | 1ull << 46 | 2ull << 61;
}

// ---- row tiles ------------------------------------------------------------------------------------------

// Tiles of up to 128 rows of the groups, by expert, so that tiles with the same weights follow one another. One CTA.
__global__ void __launch_bounds__(1024) plan_kernel(int R, int E, int groups, const int32_t* __restrict__ offsets,
                                                    int4* __restrict__ plan, int32_t* __restrict__ status) {
  __shared__ int warp_sum[32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per = groups / E;
  bool bad = false;
  for (int g = threadIdx.x; g <= groups; g += 1024) {
    const int v = offsets[g];
    bad |= v < 0 || v > R || (g > 0 && offsets[g - 1] > v);
  }
  bad = __syncthreads_or(bad);
  int base = 0;
  for (int q0 = 0; q0 < groups && !bad; q0 += 1024) {
    const int q = q0 + threadIdx.x, e = q / per;
    const int2 span = q < groups ? rows_of_group(offsets, (q - e * per) * E + e, R) : make_int2(0, 0);
    const int tiles = (span.y - span.x + BM - 1) / BM;
    int incl = tiles;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(FULL, incl, o);
      if (lane >= o) incl += v;
    }
    if (lane == 31) warp_sum[warp] = incl;
    __syncthreads();
    int before = base, all = base;
    for (int w = 0; w < 32; ++w) {
      before += w < warp ? warp_sum[w] : 0;
      all += warp_sum[w];
    }
    for (int i = 0; i < tiles; ++i)
      plan[1 + before + incl - tiles + i] = make_int4(span.x + i * BM, min(BM, span.y - span.x - i * BM), e, 0);
    base = all;
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    plan[0] = make_int4(bad ? 0 : base, !bad, 0, 0);
    *status = bad ? MOESCHED_ST_BAD_INPUT : MOESCHED_ST_OK;
  }
}

// ---- the products ---------------------------------------------------------------------------------------

struct Tile {
  int row, rows, e, n;      // rows of the result, expert, first column
  int which;                // DWEIGHT: 0 gate, 1 up, 2 down
};

template <int MODE>
__device__ __forceinline__ int tile_total(const GemmArgs& a, const int4 head) {
  if constexpr (MODE == DWEIGHT) {
    const int gu = ((a.I + BM - 1) / BM) * ((a.D + BN - 1) / BN), dn = ((a.D + BM - 1) / BM) * ((a.I + BN - 1) / BN);
    return head.y ? a.E * (2 * gu + dn) : 0;
  } else {
    const int cols = MODE == GLU || MODE == DHIDDEN ? a.I : a.D, wide = MODE == GLU ? BN / 2 : BN;
    return head.x * ((cols + wide - 1) / wide);
  }
}
template <int MODE>
__device__ __forceinline__ Tile tile_at(const GemmArgs& a, const int4 head, int t) {
  Tile w;
  if constexpr (MODE == DWEIGHT) {
    const int gu = ((a.I + BM - 1) / BM) * ((a.D + BN - 1) / BN), dn = ((a.D + BM - 1) / BM) * ((a.I + BN - 1) / BN);
    const int each = 2 * gu + dn;
    w.e = t / each;
    t -= w.e * each;
    w.which = t < gu ? 0 : t < 2 * gu ? 1 : 2;
    t -= w.which * gu;
    const int M = w.which < 2 ? a.I : a.D, m_tiles = (M + BM - 1) / BM;
    w.row = t % m_tiles * BM;
    w.rows = min(BM, M - w.row);
    w.n = t / m_tiles * BN;
  } else {
    const int cols = MODE == GLU || MODE == DHIDDEN ? a.I : a.D, wide = MODE == GLU ? BN / 2 : BN;
    const int n_tiles = (cols + wide - 1) / wide;
    const int block = t / (RASTER * n_tiles), first = block * RASTER, high = min(RASTER, head.x - first);
    t -= first * n_tiles;
    const int4 row = a.plan[1 + first + t % high];
    w.row = row.x, w.rows = row.y, w.e = row.z, w.n = t / high * wide, w.which = 0;
  }
  return w;
}
// calls f(k-block's first row or column, what it holds (64 or less), which operands) for every block of the contraction
template <int MODE, typename F>
__device__ __forceinline__ bool each_block(const GemmArgs& a, const Tile& w, F&& f) {
  if constexpr (MODE == DWEIGHT) {
    for (int g = w.e; g < a.groups; g += a.E) {
      const int2 span = rows_of_group(a.offsets, g, a.R);
      for (int r = span.x; r < span.y; r += BK)
        if (!f(r, min(BK, span.y - r), w.which)) return false;
    }
  } else {
    const int K = MODE == GLU || MODE == DHIDDEN ? a.D : a.I;
    for (int part = 0; part < (MODE == DINPUT ? 2 : 1); ++part)
      for (int k = 0; k < K; k += BK)
        if (!f(k, BK, part)) return false;
  }
  return true;
}

template <int MODE, typename T, int ACT>
__global__ void __launch_bounds__(GEMM_THREADS, 1) gemm_kernel(const __grid_constant__ GemmArgs a) {
  constexpr bool A_T = MODE == DWEIGHT, B_T = MODE == DHIDDEN || MODE == DINPUT || MODE == DWEIGHT;
  extern __shared__ unsigned char raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  unsigned long long* bars = reinterpret_cast<unsigned long long*>(smem + STAGES * STAGE_BYTES);
  const unsigned ring = smem_addr(smem);
  const unsigned full = smem_addr(bars), empty = full + 8 * STAGES, fixed = empty + 8 * STAGES, done = fixed + 8 * STAGES,
                 free_ = done + 16, drain = free_ + 16;
  int* words = reinterpret_cast<int*>(bars + 3 * STAGES + 5);
  volatile int* failed = words;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;

  if (threadIdx.x == 0) {
    *failed = 0;
    for (int s = 0; s < STAGES; ++s) {
      barrier_init(full + 8 * s, 1);
      barrier_init(empty + 8 * s, 1);
      barrier_init(fixed + 8 * s, 1);
    }
    for (int q = 0; q < 2; ++q) {
      barrier_init(done + 8 * q, 1);
      barrier_init(free_ + 8 * q, 4);
    }
    barrier_init(drain, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(words + 1)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const unsigned tmem = *reinterpret_cast<volatile unsigned*>(words + 1);
  const int4 head = a.plan[0];
  const int total = tile_total<MODE>(a, head);

  if (warp == 0) {
    if (lane == 0) {
      int stage = 0, issued = 0;
      unsigned phase = 0;
      bool ok = true;
      for (int t = blockIdx.x; t < total && ok; t += gridDim.x) {
        const Tile w = tile_at<MODE>(a, head, t);
        ok = each_block<MODE>(a, w, [&](int k, int, int part) {
          if (!barrier_wait(empty + 8 * stage, phase ^ 1, failed)) return false;
          const unsigned bar = full + 8 * stage, to = ring + stage * STAGE_BYTES, tb = to + A_BYTES;
          barrier_expect(bar, STAGE_BYTES);
          if constexpr (A_T) {
            for (int q = 0; q < 2; ++q) tma_load(to + q * MAP_BOX_BYTES, &a.a[part], bar, w.row + 64 * q, k, 0);
          } else {
            tma_load(to, &a.a[MODE == DINPUT ? part : 0], bar, k, w.row, 0);
          }
          if constexpr (MODE == GLU) {
            tma_load(tb, &a.b[0], bar, k, w.n, w.e);
            tma_load(tb + B_BYTES / 2, &a.b[1], bar, k, w.n, w.e);
          } else if constexpr (MODE == DOWN) {
            tma_load(tb, &a.b[0], bar, k, w.n, w.e);
            tma_load(tb + B_BYTES / 2, &a.b[0], bar, k, w.n + 128, w.e);
          } else {
            for (int q = 0; q < 4; ++q)
              tma_load(tb + q * MAP_BOX_BYTES, &a.b[MODE == DHIDDEN ? 0 : part], bar, w.n + 64 * q, k, MODE == DWEIGHT ? 0 : w.e);
          }
          ++issued;
          if (++stage == STAGES) stage = 0, phase ^= 1;
          return true;
        });
      }
      if (!ok) {                                            // nothing may land in shared memory that is no longer ours
        for (int q = max(0, issued - STAGES); q < issued; ++q) {
          int never = 0;
          barrier_wait(full + 8 * (q % STAGES), q / STAGES & 1, &never);
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      constexpr unsigned FORMAT = std::is_same_v<T, __half> ? 0 : 1;
      constexpr unsigned IDESC = 1u << 4 | FORMAT << 7 | FORMAT << 10 | (A_T ? 1u : 0u) << 15 | (B_T ? 1u : 0u) << 16 |
                                 (BN / 8) << 17 | (BM / 16) << 24;
      int stage = 0, slot = 0;
      unsigned phase = 0, slot_phase = 0, fixed_phase = 0;
      bool ok = true;
      for (int t = blockIdx.x; t < total && ok; t += gridDim.x) {
        const Tile w = tile_at<MODE>(a, head, t);
        bool first = true;
        const unsigned d = tmem + slot * BN;
        ok = each_block<MODE>(a, w, [&](int, int held, int) {
          if (first && !barrier_wait(free_ + 8 * slot, slot_phase ^ 1, failed)) return false;
          if (MODE == DWEIGHT && held < BK) {
            if (!barrier_wait(fixed + 8 * stage, fixed_phase >> stage & 1, failed)) return false;
            fixed_phase ^= 1u << stage;
          } else if (!barrier_wait(full + 8 * stage, phase, failed)) {
            return false;
          }
          fence_after();
          const unsigned at = ring + stage * STAGE_BYTES;
          const unsigned long long da = operand(at, A_T), db = operand(at + A_BYTES, B_T);
          const int steps = MODE == DWEIGHT ? (held + 15) / 16 : BK / 16;
          for (int s = 0; s < steps; ++s) {
            // 16 k: 32 bytes of a row, or 16 rows of 128 bytes
            mma_issue(d, da + s * (A_T ? 2048 >> 4 : 32 >> 4), db + s * (B_T ? 2048 >> 4 : 32 >> 4), IDESC, !first || s > 0);
          }
          first = false;
          mma_commit(empty + 8 * stage);
          if (++stage == STAGES) stage = 0, phase ^= 1;
          return true;
        });
        if (!first) {
          mma_commit(done + 8 * slot);
          if (++slot == 2) slot = 0, slot_phase ^= 1;
        }
      }
      if (!ok) {
        mma_commit(drain);
        int never = 0;
        barrier_wait(drain, 0, &never);
      }
    }
  } else if (warp == 2) {
    if constexpr (MODE == DWEIGHT) {                        // zeroes what a block holds behind its group's last row
      int stage = 0;
      unsigned phase = 0;
      bool ok = true;
      for (int t = blockIdx.x; t < total && ok; t += gridDim.x) {
        const Tile w = tile_at<MODE>(a, head, t);
        ok = each_block<MODE>(a, w, [&](int, int held, int) {
          // (every block is waited for: a parity says nothing about a phase that is two ahead)
          if (!__all_sync(FULL, barrier_wait(full + 8 * stage, phase, failed))) return false;
          if (held < BK) {
            const int to = (held + 15) / 16 * 16, bytes16 = (to - held) * 8;
            for (int q = lane; q < 6 * bytes16; q += 32) {
              const int box = q / bytes16, at = q - box * bytes16;
              *reinterpret_cast<uint4*>(smem + stage * STAGE_BYTES + box * MAP_BOX_BYTES + held * 128 + at * 16) = make_uint4(0, 0, 0, 0);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) barrier_arrive(fixed + 8 * stage);
          }
          if (++stage == STAGES) stage = 0, phase ^= 1;
          return true;
        });
      }
    }
  } else if (warp >= 4) {
    const int quarter = warp - 4, row = quarter * 32 + lane;
    const unsigned mine = tmem + ((unsigned)quarter << 21);
    int slot = 0;
    unsigned slot_phase = 0;
    for (int t = blockIdx.x; t < total; t += gridDim.x) {
      const Tile w = tile_at<MODE>(a, head, t);
      bool any = true;
      if constexpr (MODE == DWEIGHT) {
        any = false;
        each_block<MODE>(a, w, [&](int, int, int) { any = true; return false; });
      }
      if (any) {
        if (!__all_sync(FULL, barrier_wait(done + 8 * slot, slot_phase, failed))) break;
        fence_after();
      }
      const unsigned d = mine + slot * BN;
      const bool in = row < w.rows;
      if constexpr (MODE == GLU || MODE == DHIDDEN) {
        const size_t at = (size_t)(w.row + row) * a.I + w.n;
        constexpr int COLS = MODE == GLU ? BN / 2 : BN;
#pragma unroll 1
        for (int c = 0; c < COLS; c += 32) {
          float p[32], q[32];
          tmem_load32(d + c, p);
          if constexpr (MODE == GLU) tmem_load32(d + COLS + c, q);
          tmem_load_wait();
#pragma unroll
          for (int s = 0; s < 32; s += 8) {
            if (!in || w.n + c + s >= a.I) continue;
            if constexpr (MODE == GLU) {
              unsigned h[4], g[4], u[4];
#pragma unroll
              for (int v = 0; v < 4; ++v) {
                const int i = s + 2 * v;
                h[v] = Pair<T>::from_float(activation<ACT>(p[i]) * q[i], activation<ACT>(p[i + 1]) * q[i + 1]);
                g[v] = Pair<T>::from_float(p[i], p[i + 1]);
                u[v] = Pair<T>::from_float(q[i], q[i + 1]);
              }
              *reinterpret_cast<uint4*>(static_cast<T*>(a.out[0]) + at + c + s) = make_uint4(h[0], h[1], h[2], h[3]);
              if (a.out[1] != nullptr) {
                *reinterpret_cast<uint4*>(static_cast<T*>(a.out[1]) + at + c + s) = make_uint4(g[0], g[1], g[2], g[3]);
                *reinterpret_cast<uint4*>(static_cast<T*>(a.out[2]) + at + c + s) = make_uint4(u[0], u[1], u[2], u[3]);
              }
            } else {
              const uint4 gv = *reinterpret_cast<const uint4*>(static_cast<const T*>(a.in[0]) + at + c + s);
              const uint4 uv = *reinterpret_cast<const uint4*>(static_cast<const T*>(a.in[1]) + at + c + s);
              const unsigned gw[4] = {gv.x, gv.y, gv.z, gv.w}, uw[4] = {uv.x, uv.y, uv.z, uv.w};
              unsigned h[4], g[4], u[4];
#pragma unroll
              for (int v = 0; v < 4; ++v) {
                const float2 gate = Pair<T>::to_float(gw[v]), up = Pair<T>::to_float(uw[v]);
                const float x0 = p[s + 2 * v], x1 = p[s + 2 * v + 1];
                float f0, s0, f1, s1;
                activation_slope<ACT>(gate.x, f0, s0);
                activation_slope<ACT>(gate.y, f1, s1);
                h[v] = Pair<T>::from_float(f0 * up.x, f1 * up.y);
                g[v] = Pair<T>::from_float(x0 * up.x * s0, x1 * up.y * s1);
                u[v] = Pair<T>::from_float(x0 * f0, x1 * f1);
              }
              *reinterpret_cast<uint4*>(static_cast<T*>(a.out[0]) + at + c + s) = make_uint4(h[0], h[1], h[2], h[3]);
              *reinterpret_cast<uint4*>(static_cast<T*>(a.out[1]) + at + c + s) = make_uint4(g[0], g[1], g[2], g[3]);
              *reinterpret_cast<uint4*>(static_cast<T*>(a.out[2]) + at + c + s) = make_uint4(u[0], u[1], u[2], u[3]);
            }
          }
        }
      } else {
        const int cols = MODE == DWEIGHT && w.which == 2 ? a.I : a.D;
        const size_t first = MODE == DWEIGHT ? (size_t)w.e * a.I * a.D + (size_t)(w.row + row) * cols : (size_t)(w.row + row) * cols;
        T* out = static_cast<T*>(a.out[MODE == DWEIGHT ? w.which : 0]) + first + w.n;
#pragma unroll 1
        for (int c = 0; c < BN; c += 32) {
          float p[32];
          if (any) {
            tmem_load32(d + c, p);
            tmem_load_wait();
          } else {
#pragma unroll
            for (int s = 0; s < 32; ++s) p[s] = 0.0f;
          }
#pragma unroll
          for (int s = 0; s < 32; s += 8) {
            if (!in || w.n + c + s >= cols) continue;
            *reinterpret_cast<uint4*>(out + c + s) =
                make_uint4(Pair<T>::from_float(p[s], p[s + 1]), Pair<T>::from_float(p[s + 2], p[s + 3]),
                           Pair<T>::from_float(p[s + 4], p[s + 5]), Pair<T>::from_float(p[s + 6], p[s + 7]));
          }
        }
      }
      if (any) {
        fence_before();
        __syncwarp();
        if (lane == 0) barrier_arrive(free_ + 8 * slot);
        if (++slot == 2) slot = 0, slot_phase ^= 1;
      }
    }
  }
  fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *failed) *a.status = MOESCHED_ST_INTERNAL;
  if (warp == 1) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
  }
}

// ---- host -----------------------------------------------------------------------------------------------

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static cudaError_t encoder(EncodeFn* fn) {
  static EncodeFn found = nullptr;      // (every thread finds the same)
  if (found == nullptr) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult how;
    cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &how);
    if (e != cudaSuccess) return e;
    if (how != cudaDriverEntryPointSuccess || p == nullptr) return cudaErrorNotSupported;
    found = reinterpret_cast<EncodeFn>(p);
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
  const size_t table = ((size_t)R / BM + groups + 1) * sizeof(int4), rows = (size_t)R * I * 2;
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

template <int MODE, typename T>
static cudaError_t launch_gemm(const GemmArgs& args, int act, long long tiles, cudaStream_t stream) {
  const auto kern = (MODE == GLU || MODE == DHIDDEN) && act == MOESCHED_ACT_GELU ? gemm_kernel<MODE, T, MOESCHED_ACT_GELU>
                                                                               : gemm_kernel<MODE, T, MOESCHED_ACT_SILU>;
  const size_t smem = 1024 + STAGES * STAGE_BYTES + 256;
  if (cudaError_t e = permit_shared_memory(kern, smem); e != cudaSuccess) return e;
  const long long sms = sm_count();
  kern<<<(unsigned)(tiles < sms ? tiles : sms), GEMM_THREADS, smem, stream>>>(args);
  return cudaGetLastError();
}
template <int MODE>
static cudaError_t launch_gemm(const GemmArgs& args, int dtype, int act, long long tiles, cudaStream_t stream) {
  return dtype == MOESCHED_BF16 ? launch_gemm<MODE, __nv_bfloat16>(args, act, tiles, stream)
                                : launch_gemm<MODE, __half>(args, act, tiles, stream);
}

cudaError_t run_expert_ffn(int R, int D, int I, int E, int groups, int dtype, int act, const void* x, const void* w_gate,
                           const void* w_up, const void* w_down, const int32_t* offsets, void* y, void* gate, void* up,
                           void* scratch, int32_t* status, cudaStream_t stream) {
  const ExpertScratch at = expert_scratch(R, I, groups, false);
  unsigned char* base = static_cast<unsigned char*>(scratch);
  void* hidden = base + at.hidden;
  cudaError_t e;
  if (R <= EXPERT_FEW_ROWS) {
    e = run_few(R, D, I, E, groups, 0, dtype, act, x, w_gate, nullptr, w_up, nullptr, offsets, hidden, gate, up, status, stream);
    if (e != cudaSuccess) return e;
    return run_few(R, I, D, E, groups, 0, dtype, act, hidden, w_down, nullptr, nullptr, nullptr, offsets, y, nullptr, nullptr,
                   status, stream);
  }
  EncodeFn encode;
  if ((e = encoder(&encode)) != cudaSuccess) return e;
  int4* plan = reinterpret_cast<int4*>(base + at.plan);
  GemmArgs first = {}, second = {};
  first.plan = second.plan = plan;
  first.offsets = second.offsets = offsets;
  first.R = second.R = R, first.D = second.D = D, first.I = second.I = I, first.E = second.E = E;
  first.groups = second.groups = groups;
  first.status = second.status = status;
  if ((e = make_map(encode, &first.a[0], dtype, x, D, R, 1, BM)) != cudaSuccess) return e;
  if ((e = make_map(encode, &first.b[0], dtype, w_gate, D, I, E, BN / 2)) != cudaSuccess) return e;
  if ((e = make_map(encode, &first.b[1], dtype, w_up, D, I, E, BN / 2)) != cudaSuccess) return e;
  first.out[0] = hidden, first.out[1] = gate, first.out[2] = up;
  if ((e = make_map(encode, &second.a[0], dtype, hidden, I, R, 1, BM)) != cudaSuccess) return e;
  if ((e = make_map(encode, &second.b[0], dtype, w_down, I, D, E, BN / 2)) != cudaSuccess) return e;
  second.out[0] = y;
  plan_kernel<<<1, 1024, 0, stream>>>(R, E, groups, offsets, plan, status);
  if ((e = cudaGetLastError()) != cudaSuccess) return e;
  const long long m_tiles = (long long)R / BM + (groups < R ? groups : R);
  if ((e = launch_gemm<GLU>(first, dtype, act, m_tiles * ((I + BN / 2 - 1) / (BN / 2)), stream)) != cudaSuccess) return e;
  return launch_gemm<DOWN>(second, dtype, act, m_tiles * ((D + BN - 1) / BN), stream);
}

cudaError_t run_expert_backward(int R, int D, int I, int E, int groups, int dtype, int act, const void* dy, const void* x,
                                const void* w_gate, const void* w_up, const void* w_down, const int32_t* offsets,
                                const void* gate, const void* up, void* dx, void* dw_gate, void* dw_up, void* dw_down,
                                void* scratch, int32_t* status, cudaStream_t stream) {
  cudaError_t e;
  const size_t weights = (size_t)E * I * D * 2;
  if (R == 0) {                                             // no rows: no tensor maps, and gradients of nothing
    if ((e = cudaMemsetAsync(dw_gate, 0, weights, stream)) != cudaSuccess) return e;
    if ((e = cudaMemsetAsync(dw_up, 0, weights, stream)) != cudaSuccess) return e;
    if ((e = cudaMemsetAsync(dw_down, 0, weights, stream)) != cudaSuccess) return e;
    plan_kernel<<<1, 1024, 0, stream>>>(R, E, groups, offsets, static_cast<int4*>(scratch), status);
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
  auto map = [&](CUtensorMap* m, const void* p, int cols, int rows, int deep, int high) {
    if (e == cudaSuccess) e = make_map(encode, m, dtype, p, cols, rows, deep, high);
  };
  map(&args[0].a[0], dy, D, R, 1, BM);
  map(&args[0].b[0], w_down, I, D, E, BK);
  args[0].in[0] = gate, args[0].in[1] = up;
  args[0].out[0] = hidden, args[0].out[1] = d_gate, args[0].out[2] = d_up;
  map(&args[1].a[0], d_gate, I, R, 1, BM);
  map(&args[1].a[1], d_up, I, R, 1, BM);
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
  plan_kernel<<<1, 1024, 0, stream>>>(R, E, groups, offsets, plan, status);
  if ((e = cudaGetLastError()) != cudaSuccess) return e;
  const long long m_tiles = (long long)R / BM + (groups < R ? groups : R);
  if ((e = launch_gemm<DHIDDEN>(args[0], dtype, act, m_tiles * ((I + BN - 1) / BN), stream)) != cudaSuccess) return e;
  if ((e = launch_gemm<DINPUT>(args[1], dtype, act, m_tiles * ((D + BN - 1) / BN), stream)) != cudaSuccess) return e;
  const long long gu = (long long)((I + BM - 1) / BM) * ((D + BN - 1) / BN), dn = (long long)((D + BM - 1) / BM) * ((I + BN - 1) / BN);
  return launch_gemm<DWEIGHT>(args[2], dtype, act, E * (2 * gu + dn), stream);
}

}  // namespace moesched
