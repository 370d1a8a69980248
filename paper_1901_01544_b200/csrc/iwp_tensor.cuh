// iwp_tensor.cuh - products of 16-bit matrices on the tensor cores of sm_100a, for the output head of iwp_head.cuh.
//
// One persistent kernel template: C[M, N] = A[M, K] B[N, K]^T with fp32 accumulators in tensor memory, and what
// becomes of a finished tile left to an epilogue class.  Either operand may lie K-contiguous or M/N-contiguous
// in memory (the tensor cores read both), so none of the three products of a head is ever transposed, and the two
// gradients, which need nothing of each other, are one launch with two problems.
//
// A CTA pair (cta_group::2) works on one 256 x 256 tile: each CTA stages its own 128 rows of A and 128 rows of B, so
// that every byte brought into shared memory feeds twice the arithmetic of a single CTA's 128 x 256 tile
// (64 instead of 96 bytes per SM and clock at the full tensor rate).  Problems with few tiles take tiles of 128 or
// 64 columns instead (pick_tile_n).  Roles per CTA: warp 0 issues the tile loads (TMA), warp 1 of the pair's first
// CTA issues the products, warp 2 owns the tensor memory, warps 4..11 are the epilogue (warp % 4 = the 32 lanes of
// tensor memory it may read, the other half of the columns for warps 8..11).  Two accumulator tiles of 256 columns
// fill the 512 columns of tensor memory, so the epilogue of one tile runs beside the products of the next.
//
// Bound by the tensor cores for K of about 1000 and more, and there by power: the logits of 8192 x 131072 x 4096 take 5.6 ms
// alone (1.57 PFLOP/s), its two gradients 13.0 ms (1.35), in a loop both settle near 1.3, as a library product does
// (1.37). 1024 x 50176 x 1024: logits 70 us (1.5 PFLOP/s; 80 with codes), dhidden 84, dweight 87. Below K of 500
// an epilogue (7000 clocks for 256 x 256 logits with their exponentials) takes longer than a tile's products.
//
// Every wait is bounded: a wait that runs out sets the status word and marks the CTA dead; the roles then fall
// through to the common end, which gives copies in flight time to land, frees the tensor memory and returns.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/iwp.h"

namespace iwp_tc {

constexpr int TILE_M = 128;    // rows of a CTA's accumulator (lanes of tensor memory)
constexpr int TILE_N = 256;    // columns of the accumulator
constexpr int BLOCK_K = 64;    // elements of K per stage: 128 bytes, one swizzle row
constexpr int EPI_WARPS = 8;
constexpr int THREADS = 128 + 32 * EPI_WARPS;
constexpr int STAGING_BYTES = 32 * 128;                 // per epilogue warp: a row of 128 bytes per lane
constexpr uint32_t WAIT_TRIES = 1u << 18;               // x 20 us at most per try: about 5 s
constexpr uint32_t WAIT_HINT_NS = 20000;

constexpr int CG = 2;                               // CTAs per tile
constexpr int A_BYTES = TILE_M * BLOCK_K * 2;
constexpr int MAX_STAGES = 8;
constexpr int WIDE_STAGE = A_BYTES + TILE_N / CG * BLOCK_K * 2;
// Shared memory: a ring of load stages (6 of the widest tiles, 5 beside an epilogue with two staging areas per warp; more
// of narrower tiles), the staging areas, barriers.
__host__ __device__ constexpr int ring_bytes(int areas) { return (areas == 2 ? 5 : 6) * WIDE_STAGE; }
__host__ __device__ constexpr int smem_bytes(int areas) { return 1024 + ring_bytes(areas) + areas * EPI_WARPS * STAGING_BYTES + 256; }
static_assert(smem_bytes(1) <= 227 * 1024 && smem_bytes(2) <= 227 * 1024, "shared memory of a CTA");

// The 16-byte word `word` (0..7) of staging row `row`: rotated by the row, so that neither lanes that write their own
// rows nor lanes that read neighbouring words of a row meet in a bank.
__device__ __forceinline__ char* staged(char* staging, int row, int word) { return staging + 128 * row + 16 * (word ^ (row & 7)); }

// ---- small wrappers of the instructions used ---------------------------------------------------------

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}

// the address, in the cluster's shared window, of `addr` in the CTA `rank` of this cluster
__device__ __forceinline__ uint32_t map_to(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}

__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

// What these barriers order is tensor memory and asynchronous copies, which have their own fences; a release at cluster
// scope would wait for every store of the epilogue besides.
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t cluster_bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}

__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity), "r"(WAIT_HINT_NS)
      : "memory");
  return ok != 0;
}

// Bounded wait; false = gave up (or another role of this CTA did).
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int* dead, int* status, uint32_t tries = WAIT_TRIES) {
  if (mbar_try(bar, parity)) return true;
  for (uint32_t i = 0; i < tries; i++) {
    if (mbar_try(bar, parity)) return true;
    if (*dead) return false;
  }
  *dead = 1;
  atomicExch(status, IWP_ERR_TIMEOUT);
  return false;
}

#ifdef IWP_DEBUG_CHECKS
// For the test of the waits: two warps wait for a barrier that nothing arrives on, one of them at most 40 ms.
__global__ void __launch_bounds__(64) k_wait_probe(int* status, int* gave_up) {
  __shared__ uint64_t bar;
  __shared__ volatile int dead;
  if (threadIdx.x == 0) {
    mbar_init(smem_u32(&bar), 1);
    dead = 0;
  }
  __syncthreads();
  if (threadIdx.x % 32 == 0 && !mbar_wait(smem_u32(&bar), 0, &dead, status, threadIdx.x == 0 ? 2000u : WAIT_TRIES)) atomicAdd(gave_up, 1);
}
#endif

__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(bar)
      : "memory");
}

__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}

// Arrives on the barrier at this offset in both CTAs of the pair once all products issued so far are done.
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
               "h"(static_cast<uint16_t>(3))
               : "memory");
}

// Programmatic launches: a kernel may start while the one before it drains, and touches memory only after wait().
__device__ __forceinline__ void launch_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// 2^x, denormal results flushed (their weight in any sum here is below its last bit)
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }

// Two floats at a time: sm_100's packed arithmetic, where issue slots count.
using f2 = unsigned long long;
__device__ __forceinline__ f2 pack(float a, float b) {
  f2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 unpack(f2 x) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
  return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
  f2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
  f2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
  f2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// 32 columns of this warp's 32 lanes: v[j] = column j of the lane's row.
__device__ __forceinline__ void tmem_load32(uint32_t addr, float (&v)[32]) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr)
      : "memory");
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int j = 0; j < 32; j++) v[j] = __uint_as_float(r[j]);
}

// Shared-memory operand descriptor, 128-byte swizzle.  K-contiguous operands: rows of 128 bytes, groups of 8 rows
// every 1024 bytes.  M/N-contiguous operands: blocks of 64 rows of M/N (128 bytes) x BLOCK_K, one block after the
// other (the leading offset), groups of 8 along K every 1024 bytes.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, bool k_contiguous) {
  const uint64_t lead = k_contiguous ? 1 : (BLOCK_K * 128) >> 4;
  return static_cast<uint64_t>((addr & 0x3FFFF) >> 4) | (lead << 16) | (static_cast<uint64_t>(1024 >> 4) << 32) | (1ull << 46) |
         (2ull << 61);
}

// ---- the work list ---------------------------------------------------------------------------------

struct Problem {
  CUtensorMap a, b;
  int m_tiles, n_tiles;  // tiles of CG * TILE_M rows and tile_n columns
  int tile_n;            // 256, 128 or 64
  int k_blocks;          // blocks of BLOCK_K along K
  int splits;            // the K range in this many parts (each part a tile of its own)
  int seg;               // blocks of K per accumulator
  uint32_t idesc;
  int a_kc, b_kc;        // which operands are K-contiguous
  CUtensorMap b_other;   // what takes B's place if *use_other (on the device; NULL: never), last problem of a launch only
  const int* use_other;
};

// Up to two problems over the pairs of a launch.  Every pair first takes `rounds` tiles of problem 0; the first `rest`
// pairs take one more each, and the others meanwhile `fill` tiles of problem 1 each; what is left of problem 1 is dealt
// round by round.  (The tiles of one problem all cost the same, so the host can balance this without a counter.)
template <int N>
struct Problems {
  Problem p[N];
  int rounds, rest, fill;
  int stages, b_bytes;  // of the ring in shared memory, and B's share of a stage
  int early;  // 1: the operands were complete before the kernel in front of this one let it start, so that only the
              // epilogue has to wait for that kernel's end
  int* status;
};

struct Tile {
  int p, m, n, split, k0, k1;
};

template <int N>
__device__ __forceinline__ void deal(const Problems<N>& w, int pair, int pairs, int step, int& p, int& i) {
  p = 0;
  if constexpr (N == 1) {
    i = step * pairs + pair;
    return;
  }
  if (step < w.rounds) {
    i = step * pairs + pair;
    return;
  }
  step -= w.rounds;
  if (w.rest > 0) {
    if (pair < w.rest) {
      if (step == 0) {
        i = w.rounds * pairs + pair;
        return;
      }
      step -= 1;
    } else {
      p = 1;
      i = step * (pairs - w.rest) + pair - w.rest;
      if (step < w.fill) return;
      step -= w.fill;
    }
  }
  p = 1;
  i = step * pairs + pair;
  if (w.rest > 0) i += w.fill * (pairs - w.rest) - w.rest + (pair < w.rest ? pairs : 0);  // the pairs without one go first
}

// The tile of a pair's step; false = it has no more.  Tiles of one problem in groups of up to 16 of the shorter side, so
// that the tiles in flight share operands in the L2.
template <int N>
__device__ __forceinline__ bool tile_at(const Problems<N>& w, int pair, int pairs, int step, Tile& t) {
  int i;
  deal(w, pair, pairs, step, t.p, i);
  const Problem& q = w.p[t.p];
  const int per = q.m_tiles * q.n_tiles;
  if (i >= per * q.splits) return false;
  t.split = i / per;
  const int r = i - t.split * per;
  const bool m_short = q.m_tiles <= q.n_tiles;
  const int s = m_short ? q.m_tiles : q.n_tiles, l = m_short ? q.n_tiles : q.m_tiles;
  const int g = r / (16 * l);
  const int size = min(16, s - 16 * g);
  const int o = r - g * 16 * l;
  const int x = 16 * g + o % size, y = o / size;
  t.m = m_short ? x : y;
  t.n = m_short ? y : x;
  t.k0 = static_cast<int>(static_cast<int64_t>(q.k_blocks) * t.split / q.splits);
  t.k1 = static_cast<int>(static_cast<int64_t>(q.k_blocks) * (t.split + 1) / q.splits);
  return true;
}

// Epi (device class): `Args`; AREAS, the staging areas per warp; begin(args, where), before the tile is there; tile(args,
// where, begun, sums), in which an epilogue warp disposes of its 32 rows and half of the tile's columns.
//
// Tensor cores cut what a term loses against the running sum, so long sums of one sign come out low: with K = 131072 by up to
// 1.4e-3 of themselves, with 8192 by 1.5e-5, 1024 by 1e-6.  With SUMS the tensor memory is therefore emptied into registers
// every `seg` blocks of K (at most 1024 elements) and added up there, in fp32 rounded to nearest, while the products go on in
// the other accumulator; tile() gets an array of pairs of columns.  (dhidden of 1024 x 50176 x 1024: 84 us, 78 without;
// segments of 4096 take the same.)  Without, for K of one segment, it gets an address in tensor memory.
struct Where {
  int row0;     // first of the warp's 32 rows; the lane's row is row0 + lane
  int col0;     // first of the warp's columns
  int width;    // number of them: half a tile
  int lane, p, split;
  char* staging;  // Epi::AREAS areas of STAGING_BYTES
  int area;       // the one to use next, for epilogues that take turns
};

template <int N, class Epi>
__global__ void __launch_bounds__(THREADS, 1)
    k_product(const __grid_constant__ Problems<N> w, const __grid_constant__ typename Epi::Args args) {
  extern __shared__ char smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  char* const smem = smem_raw + (((raw + 1023) & ~1023u) - raw);  // the same offset in both CTAs of a pair
  const uint32_t base = smem_u32(smem);
  char* const staging = smem + ring_bytes(Epi::AREAS);
  char* const ctl = staging + Epi::AREAS * EPI_WARPS * STAGING_BYTES;
  const uint32_t bars = smem_u32(ctl);
  const uint32_t full = bars, empty = bars + 8 * MAX_STAGES, acc_full = empty + 8 * MAX_STAGES, acc_empty = acc_full + 16;
  volatile int* const dead = reinterpret_cast<volatile int*>(ctl + 8 * (2 * MAX_STAGES + 4));
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(ctl + 8 * (2 * MAX_STAGES + 4) + 4);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  launch_next();
  if (threadIdx.x == 0) {
    for (int s = 0; s < w.stages; s++) {
      mbar_init(full + 8 * s, 1);
      mbar_init(empty + 8 * s, 1);
    }
    for (int b = 0; b < 2; b++) {
      mbar_init(acc_full + 8 * b, 1);
      mbar_init(acc_empty + 8 * b, CG * EPI_WARPS);
    }
    *dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
#pragma unroll
    for (int p = 0; p < N; p++)
      if (w.p[p].n_tiles) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&w.p[p].a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&w.p[p].b) : "memory");
      }
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(tmem_slot)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    fence_before();
  }
  __syncthreads();
  cluster_sync();
  fence_after();
  const uint32_t tmem = *tmem_slot;
  if (!w.early || warp >= 4) wait_previous();

  const int pair = blockIdx.x / CG, pairs = gridDim.x / CG;
  const int stages = w.stages, stage_bytes = A_BYTES + w.b_bytes;
  Tile t;

  // An epilogue that sums holds 128 columns per thread: 88 registers for each thread of the first four warps, 208 for
  // the eight epilogue warps, of the 384 x 168 that the block was launched with.
  if (warp < 4) {
    if constexpr (Epi::SUMS) asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == 0 && lane == 0) {  // ---- loads
      int s = 0;
      uint32_t phase = 0;
      const uint32_t full_of_pair = map_to(full, 0);  // both CTAs' loads are counted by the first CTA
      const bool other = w.p[N - 1].use_other && __ldcg(w.p[N - 1].use_other);
      for (int i = 0; !*dead && tile_at(w, pair, pairs, i, t); i++) {
        const Problem& q = w.p[t.p];
        const int rows_b = q.tile_n / CG;
        const int row_a = t.m * TILE_M * CG + static_cast<int>(rank) * TILE_M;
        const int row_b = t.n * q.tile_n + static_cast<int>(rank) * rows_b;
        const bool a_kc = q.a_kc, b_kc = q.b_kc;
        const CUtensorMap* const map_b = other && t.p == N - 1 ? &q.b_other : &q.b;
        // an M/N-contiguous box is 64 columns wide even where a CTA needs 32 of them
        const uint32_t bytes = CG * (A_BYTES + (b_kc ? rows_b : max(rows_b, 64)) * BLOCK_K * 2);
        for (int kb = t.k0; kb < t.k1; kb++) {
          if (!mbar_wait(empty + 8 * s, phase ^ 1, dead, w.status)) break;
          if (rank == 0) mbar_expect(full + 8 * s, bytes);
          const uint32_t bar = full_of_pair + 8 * s;
          const uint32_t at_a = base + s * stage_bytes, at_b = at_a + A_BYTES;
          if (a_kc) {
            tma_load(at_a, &q.a, kb * BLOCK_K, row_a, bar);
          } else {
            tma_load(at_a, &q.a, row_a, kb * BLOCK_K, bar);
            tma_load(at_a + 64 * 128, &q.a, row_a + 64, kb * BLOCK_K, bar);
          }
          if (b_kc) {
            tma_load(at_b, map_b, kb * BLOCK_K, row_b, bar);
          } else {
            tma_load(at_b, map_b, row_b, kb * BLOCK_K, bar);
            if (rows_b > 64) tma_load(at_b + 64 * 128, map_b, row_b + 64, kb * BLOCK_K, bar);
          }
          if (++s == stages) {
            s = 0;
            phase ^= 1;
          }
        }
      }
    } else if (warp == 1 && lane == 0 && rank == 0) {  // ---- products
      int s = 0, b = 0;
      uint32_t phase = 0, acc_phase = 0;
      for (int i = 0; !*dead && tile_at(w, pair, pairs, i, t); i++) {
        const Problem& q = w.p[t.p];
        // 16 elements of K further: 32 bytes along a K-contiguous row, 16 rows of 128 bytes otherwise
        const bool a_kc = q.a_kc, b_kc = q.b_kc;
        const uint64_t step_a = a_kc ? 2 : 128, step_b = b_kc ? 2 : 128;
        const uint32_t idesc = q.idesc;
        for (int k0 = t.k0; k0 < t.k1; k0 += q.seg) {
          const int k1 = min(t.k1, k0 + q.seg);
          if (!mbar_wait(acc_empty + 8 * b, acc_phase ^ 1, dead, w.status)) break;
          fence_after();
          for (int kb = k0; kb < k1; kb++) {
            if (!mbar_wait(full + 8 * s, phase, dead, w.status)) break;
            fence_after();
            const uint32_t at_a = base + s * stage_bytes;
            const uint64_t da = operand_desc(at_a, a_kc), db = operand_desc(at_a + A_BYTES, b_kc);
#pragma unroll
            for (int k = 0; k < BLOCK_K / 16; k++)
              mma(tmem + b * TILE_N, da + k * step_a, db + k * step_b, idesc, (kb > k0 || k > 0) ? 1u : 0u);
            mma_commit(empty + 8 * s);
            if (++s == stages) {
              s = 0;
              phase ^= 1;
            }
          }
          mma_commit(acc_full + 8 * b);
          if (++b == 2) {
            b = 0;
            acc_phase ^= 1;
          }
        }
      }
    }
  } else {  // ---- epilogue
    if constexpr (Epi::SUMS) asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    const int e = warp - 4;
    int b = 0;
    uint32_t acc_phase = 0;
    const uint32_t empty_of_pair = map_to(acc_empty, 0);
    bool ok = true;
    Where at;
    at.area = 0;
    at.staging = staging + e * Epi::AREAS * STAGING_BYTES;
    // the accumulator's turn is over: the products may write it again
    auto release = [&] {
      fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(empty_of_pair + 8 * b);
      if (++b == 2) {
        b = 0;
        acc_phase ^= 1;
      }
    };
    // where the warp's part of a tile lies, and what its rows need from memory: fetched one tile ahead
    auto locate = [&](const Tile& t, Where& at) {
      const Problem& q = w.p[t.p];
      at.width = q.tile_n / 2;
      at.row0 = (CG * t.m + static_cast<int>(rank)) * TILE_M + (e % 4) * 32;
      at.col0 = t.n * q.tile_n + (e / 4) * at.width;
      at.p = t.p;
      at.split = t.split;
    };
    at.lane = lane;
    bool more = tile_at(w, pair, pairs, 0, t);
    Where coming = at;
    locate(t, coming);
    auto begun = Epi::begin(args, coming);
    for (int i = 1; ok && more; i++) {
      const int k0 = t.k0, k1 = t.k1, seg = w.p[t.p].seg, area = at.area;
      at = coming;
      at.area = area;
      auto now = begun;
      const uint32_t mine = tmem + (e / 4) * at.width + (static_cast<uint32_t>(e % 4) << 21);
      more = tile_at(w, pair, pairs, i, t);
      if (more) {
        locate(t, coming);
        begun = Epi::begin(args, coming);
      }
      auto wait = [&] {
        ok = __all_sync(0xFFFFFFFFu, mbar_wait(acc_full + 8 * b, acc_phase, dead, w.status));
        if (ok) fence_after();
        return ok;
      };
      if (!wait()) break;
      if constexpr (Epi::SUMS) {
        f2 acc[TILE_N / 4];
        auto segment = [&](auto first) {
#pragma unroll
          for (int c = 0; c < TILE_N / 64; c++) {
            if (32 * c < at.width) {
              float v[32];
              tmem_load32(mine + b * TILE_N + 32 * c, v);
#pragma unroll
              for (int j = 0; j < 16; j++) {
                const f2 x = pack(v[2 * j], v[2 * j + 1]);
                acc[16 * c + j] = decltype(first)::value ? x : add2(acc[16 * c + j], x);
              }
            }
          }
          release();
        };
        segment(std::true_type{});
        for (int k = k0 + seg; k < k1 && wait(); k += seg) segment(std::false_type{});
        if (ok) Epi::tile(args, at, now, acc);
      } else {
        Epi::tile(args, at, now, mine + b * TILE_N);
        release();
      }
    }
  }
  if (warp >= 4 && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");  // the epilogue's last copies
  __syncwarp();
  __syncthreads();
  if (*dead) __nanosleep(1000000);  // copies in flight land in microseconds
  cluster_sync();
  if (warp == 2) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
  }
}

__device__ __forceinline__ uint32_t pack2(float a, float b, int type) {
  if (type == 1) {
    __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t*>(&h);
  }
  __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<uint32_t*>(&h);
}

__device__ __forceinline__ float2 unpack2(uint32_t x, int type) {
  if (type == 1) return __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&x));
  return __half22float2(*reinterpret_cast<__half2*>(&x));
}

__device__ __forceinline__ float load_as_float(const void* p, int64_t i, int type) {
  if (type == 0) return static_cast<const float*>(p)[i];
  if (type == 1) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
  return __half2float(static_cast<const __half*>(p)[i]);
}

__device__ __forceinline__ void store_as(void* p, int64_t i, float v, int type) {
  if (type == 0)
    static_cast<float*>(p)[i] = v;
  else if (type == 1)
    static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
  else
    static_cast<__half*>(p)[i] = __float2half_rn(v);
}

// The warp's staging rows (32 rows of 64 16-bit columns, swizzled as `map` expects) to a matrix, by one asynchronous copy;
// rows and columns outside the matrix are dropped.  staging_free() waits until all but the last LEFT copies have read their
// rows.
template <int LEFT>
__device__ __forceinline__ void staging_free(int lane) {
  if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(LEFT) : "memory");
  __syncwarp();
}
__device__ __forceinline__ void store_staged(const CUtensorMap* map, char* staging, int row0, int col0, int lane) {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncwarp();
  if (lane == 0) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(col0), "r"(row0),
                 "r"(smem_u32(staging))
                 : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
  }
}

// A chunk of 32 columns (v: this lane's row) into the warp's staging rows, in fp32, or in 16 bits from the 16-byte word `word`
// of the row on.
__device__ __forceinline__ void stage_chunk(const float (&v)[32], char* staging, int lane) {
#pragma unroll
  for (int j = 0; j < 8; j++) *reinterpret_cast<float4*>(staged(staging, lane, j)) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
}
__device__ __forceinline__ void stage_chunk(const float (&v)[32], char* staging, int lane, int word, int type) {
#pragma unroll
  for (int j = 0; j < 4; j++)
    *reinterpret_cast<uint4*>(staged(staging, lane, word + j)) =
        make_uint4(pack2(v[8 * j], v[8 * j + 1], type), pack2(v[8 * j + 2], v[8 * j + 3], type), pack2(v[8 * j + 4], v[8 * j + 5], type),
                   pack2(v[8 * j + 6], v[8 * j + 7], type));
}

// n staged columns of 16 bits (at most 64) to a row-major matrix; rows outside are dropped, the caller synchronises the warp
// before and after.  32 columns in rows that start at multiples of 16 bytes (`wide`): 8 rows of 64 bytes at a time.  Otherwise
// one or two rows at a time in the 4-byte words of memory; of a row that starts in the middle of one, its first and its last column are
// stored on their own.
__device__ __forceinline__ void write_rows16(char* staging, uint16_t* out, int64_t ld, bool wide, int row0, int rows, int n, int lane) {
  if (wide && n == 32) {
    const int r = lane >> 2, c = lane & 3;
#pragma unroll
    for (int i = 0; i < 32; i += 8) {
      const uint4 x = *reinterpret_cast<const uint4*>(staged(staging, r + i, c));
      if (row0 + r + i < rows) *reinterpret_cast<uint4*>(out + (r + i) * ld + 8 * c) = x;
    }
    return;
  }
  auto words = [&](auto lanes) {  // of a row
    constexpr int LANES = decltype(lanes)::value, STEP = 32 / LANES;
    const int c = lane % LANES;
    uint16_t* row = out + lane / LANES * ld;
#pragma unroll 4
    for (int i = lane / LANES; i < 32; i += STEP, row += STEP * ld) {
      if (row0 + i >= rows) continue;
      const int odd = static_cast<int>(reinterpret_cast<uintptr_t>(row) >> 1 & 1), k = 2 * c + odd;
      auto at = [&](int k) { return *reinterpret_cast<const uint16_t*>(staged(staging, i, k >> 3) + 2 * (k & 7)); };
      if (k + 1 < n)
        *reinterpret_cast<uint32_t*>(row + k) = at(k) | static_cast<uint32_t>(at(k + 1)) << 16;
      else if (k < n)
        row[k] = at(k);
      if (odd && c == 0) row[0] = at(0);
    }
  };
  if (n > 32)
    words(std::integral_constant<int, 32>{});
  else
    words(std::integral_constant<int, 16>{});
}

// A chunk staged in fp32 to a row-major matrix, in whole 32-byte sectors where rows are `wide`; rows and columns outside are
// dropped.  TYPE: IWP_F32, or the 16 bits of a sum.  `add`: the old contents are added first (in fp32; all of a batch on
// their way at once, since the compiler cannot tell that a store does not touch them).  The caller synchronises the warp before
// and after.
template <int BATCH>
__device__ __forceinline__ void write_chunk(char* staging, void* out, int64_t ld, int type, bool wide, bool add, int row0, int rows, int col0,
                                            int cols, int lane) {
  const bool whole = wide && col0 + 32 <= cols;
  if (whole && type == 0) {
    const int r = lane >> 3, c = lane & 7;  // 4 rows of 128 bytes at a time
    float* p = static_cast<float*>(out) + (row0 + r) * ld + col0 + 4 * c;
#pragma unroll 1
    for (int h = 0; h < 32; h += 4 * BATCH, p += 4 * BATCH * ld) {
      float4 old[BATCH];
      if (add) {
#pragma unroll
        for (int i = 0; i < BATCH; i++)
          if (row0 + r + h + 4 * i < rows) old[i] = *reinterpret_cast<const float4*>(p + 4 * i * ld);
      }
#pragma unroll
      for (int i = 0; i < BATCH; i++) {
        float4 x = *reinterpret_cast<const float4*>(staged(staging, r + h + 4 * i, c));
        if (add) x = make_float4(x.x + old[i].x, x.y + old[i].y, x.z + old[i].z, x.w + old[i].w);
        if (row0 + r + h + 4 * i < rows) *reinterpret_cast<float4*>(p + 4 * i * ld) = x;
      }
    }
  } else if (type == 0) {  // ragged columns or unaligned rows of fp32: a row at a time
    if (col0 + lane < cols) {
      float* p = static_cast<float*>(out) + row0 * ld + col0 + lane;
#pragma unroll 1
      for (int h = 0; h < 32; h += 2 * BATCH, p += 2 * BATCH * ld) {
        float old[2 * BATCH];
        if (add) {
#pragma unroll
          for (int i = 0; i < 2 * BATCH; i++)
            if (row0 + h + i < rows) old[i] = p[i * ld];
        }
#pragma unroll
        for (int i = 0; i < 2 * BATCH; i++) {
          float x = reinterpret_cast<const float*>(staged(staging, h + i, lane >> 2))[lane & 3];
          if (add) x += old[i];
          if (row0 + h + i < rows) p[i * ld] = x;
        }
      }
    }
  } else {  // a 16-bit sum: element by element, a row at a time
    for (int i = 0; i < 32 && row0 + i < rows; i++) {
      if (col0 + lane < cols) {
        const int64_t at = (row0 + i) * ld + col0 + lane;
        const float x = reinterpret_cast<const float*>(staged(staging, i, lane >> 2))[lane & 3];
        store_as(out, at, x + load_as_float(out, at, type), type);
      }
    }
  }
}

// 32 columns of 16 bits that are packed already, staged and written; rows of 16-byte multiples, all columns inside.
__device__ __forceinline__ void store_packed(const uint32_t (&u)[16], char* staging, uint16_t* out, int64_t ld, int row0, int rows, int col0,
                                             int lane) {
#pragma unroll
  for (int j = 0; j < 4; j++) *reinterpret_cast<uint4*>(staged(staging, lane, j)) = make_uint4(u[4 * j], u[4 * j + 1], u[4 * j + 2], u[4 * j + 3]);
  __syncwarp();
  const int r = lane >> 2, c = lane & 3;  // 8 rows of 64 bytes at a time
#pragma unroll
  for (int i = 0; i < 32; i += 8) {
    const uint4 x = *reinterpret_cast<const uint4*>(staged(staging, r + i, c));
    if (row0 + r + i < rows) *reinterpret_cast<uint4*>(out + (row0 + r + i) * ld + col0 + 8 * c) = x;
  }
  __syncwarp();
}

}  // namespace iwp_tc
