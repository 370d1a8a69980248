// iwp_balance.cuh - balance loss of a router over E experts: per-expert counts, mean probabilities, loss and gradient.
//
// The gradient of a row needs the counts of the whole batch (f_e) but no other row's probabilities, so the logits are
// read once and the gradient written once.  A row lives in the registers of 1 to 32 lanes: softmax, gradient, and
// running column sums of p for the loss; a group of lanes fetches its next rows before it works on the present ones.
// Short batches (bound by latency) are one launch of one thread-block cluster, whose CTAs exchange counts and column
// sums through distributed shared memory.  Long batches (bound by memory: 2 T E elements) are two launches: counts per
// block, then the rows on every SM, whose column sums the last block to finish adds in the order of the blocks.
#pragma once

#include <cooperative_groups.h>
#include <math_constants.h>

#include "../../include/iwp_loss.h"
#include "iwp_tensor.cuh"

namespace iwp_balance {

namespace cg = cooperative_groups;

constexpr int MAX_EXPERTS = 1024;
constexpr int COUNT_BLOCKS = 128, COUNT_CLUSTER = 8, COUNT_THREADS = 512;  // 16 histograms come out of the 128 blocks
constexpr int COUNT_PARTS = COUNT_BLOCKS / COUNT_CLUSTER, MAX_CLUSTER = 16;

struct Header {
  int status;
  uint32_t ticket;  // wraps to zero with the last block of a launch
};

struct Args {
  Header* hdr;
  int* counts;
  const void* logits;
  const void* ids;
  const uint8_t* mask;
  const float* dloss;
  void* dlogits;
  int* part_counts;  // [COUNT_PARTS][E + 1]: counts, tokens; NULL: the cluster counts for itself
  float* part;       // [gridDim.x][padded(E)]
  float* loss;
  float* mean_prob;
  int64_t logits_ld, dlogits_ld, ids_ld, T;
  int E, k, ids_bytes;
  float coef, scale;
};

// Row stride of the blocks' column sums.
__host__ __device__ constexpr int padded(int E) { return (E + 3) / 4 * 4; }

// Adds the ids of tokens [t0, t1) to a histogram in shared memory (cleared by the caller) and returns this thread's share
// of the number of tokens.  L lanes (a power of two) share a token; `AHEAD` tokens are in flight per lane.
__device__ __forceinline__ int count_ids(const Args& a, int64_t t0, int64_t t1, int* hist) {
  constexpr int AHEAD = 4;
  int L = 1;
  while (L < 32 && L < a.k) L *= 2;
  const int j0 = threadIdx.x & (L - 1), stride = static_cast<int>(blockDim.x) / L;
  int n = 0;
  for (int64_t t = t0 + threadIdx.x / L; t < t1; t += AHEAD * stride) {
    for (int j = j0; j < a.k; j += L) {
      int64_t e[AHEAD];
      bool on[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; u++) {
        const int64_t at = min(t + u * stride, t1 - 1) * a.ids_ld + j;  // beyond the end: loaded again, not counted
        e[u] = a.ids_bytes == 8 ? static_cast<const int64_t*>(a.ids)[at] : static_cast<const int32_t*>(a.ids)[at];
      }
#pragma unroll
      for (int u = 0; u < AHEAD; u++) on[u] = t + u * stride < t1;
      if (a.mask) {
        uint8_t m[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; u++) m[u] = a.mask[min(t + u * stride, t1 - 1)];
#pragma unroll
        for (int u = 0; u < AHEAD; u++) on[u] = on[u] && m[u];
      }
#pragma unroll
      for (int u = 0; u < AHEAD; u++) {
        n += on[u] && j == 0;
        if (on[u] && e[u] >= 0 && e[u] < a.E) atomicAdd(&hist[e[u]], 1);
      }
    }
  }
  return n;
}

__global__ void __launch_bounds__(COUNT_THREADS) k_balance_counts(const Args a) {
  __shared__ int hist[MAX_EXPERTS + 1];
  for (int e = threadIdx.x; e <= a.E; e += blockDim.x) hist[e] = 0;
  iwp_tc::wait_previous();
  iwp_tc::launch_next();  // after the wait: whoever runs beside this kernel may read the inputs
  __syncthreads();
  const int64_t per = (a.T + gridDim.x - 1) / gridDim.x, t0 = blockIdx.x * per, t1 = min(a.T, t0 + per);
  const int n = __reduce_add_sync(0xFFFFFFFFu, count_ids(a, t0, t1, hist));
  if ((threadIdx.x & 31) == 0 && n) atomicAdd(&hist[a.E], n);
  cg::cluster_group cluster = cg::this_cluster();
  cluster.sync();
  // the blocks of a cluster share out the experts
  for (int e = cluster.block_rank() * blockDim.x + threadIdx.x; e <= a.E; e += COUNT_CLUSTER * blockDim.x) {
    int c = 0;
#pragma unroll
    for (int b = 0; b < COUNT_CLUSTER; b++) c += cluster.map_shared_rank(hist, b)[e];
    a.part_counts[blockIdx.x / COUNT_CLUSTER * (a.E + 1) + e] = c;
  }
  cluster.sync();  // nobody leaves while its counts are read
}

template <int TYPE>
struct Elem {
  using T = float;
};
template <>
struct Elem<IWP_BF16> {
  using T = __nv_bfloat16;
};
template <>
struct Elem<IWP_F16> {
  using T = __half;
};

using iwp_tc::add2;
using iwp_tc::f2;
using iwp_tc::fma2;
using iwp_tc::mul2;
using iwp_tc::pack;
using iwp_tc::unpack;

// Threads of a block, by the number of columns a lane holds (about five registers each).
__host__ __device__ constexpr int threads_of(int columns) { return columns <= 8 ? 1024 : columns <= 16 ? 512 : 256; }

constexpr int SLOTS = 4;
__host__ __device__ constexpr int slot_bytes(int columns, int size) { return SLOTS * threads_of(columns) * columns * size; }

// 131072 x 256 fp32: 56 us for 268 MB (4.8 TB/s), after 12 us of k_balance_counts on 1 M 64-bit ids; 64 x 8: 6 us in all.
//
// G lanes share a row; a lane holds N groups of VEC neighbouring columns: columns (n * G + lane) * VEC + v.
template <int TYPE, int VEC, int N>
__global__ void __launch_bounds__(threads_of(VEC* N), 1) k_balance_rows(const Args a, int G) {
  using E_t = typename Elem<TYPE>::T;
  constexpr int M = VEC * N, DEPTH = SLOTS, THREADS = threads_of(M), WARPS = THREADS / 32;
  static_assert(M % 2 == 0, "columns go in pairs");
  struct alignas(sizeof(E_t) * VEC) Pack {
    E_t x[VEC];
  };
  __shared__ int sh_mine[MAX_EXPERTS + 1], sh_count[MAX_EXPERTS + 1];
  __shared__ float sh_f[MAX_EXPERTS];
  __shared__ float sh_sum[MAX_EXPERTS];
  __shared__ float sh_loss[32];
  __shared__ bool last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane & (G - 1);
  const bool alone = a.part_counts == nullptr;

  // rows of this block's step s: from s * rows on.  A thread copies what it will need of a later step into slots of
  // its own (nobody else reads them, so no barrier): DEPTH - 1 steps are in flight.
  const int rows = THREADS / G;
  const int64_t steps = (a.T + rows - 1) / rows;
  extern __shared__ __align__(16) char sh_slots[];
  auto slot = [&](int i, int n) { return reinterpret_cast<Pack*>(sh_slots) + (i * N + n) * THREADS + tid; };
  uint32_t ons = 0;  // bit i: slot i holds a row that counts
  auto fetch = [&](int64_t step, int i) {
    const int64_t t = step * rows + tid / G;
    const bool on = step < steps && t < a.T && (!a.mask || a.mask[t]);
    ons = (ons & ~(1u << i)) | (static_cast<uint32_t>(on) << i);
    const E_t* const from = static_cast<const E_t*>(a.logits) + t * a.logits_ld + g * VEC;
#pragma unroll
    for (int n = 0; n < N; n++) {
      if (on && (n * G + g) * VEC < a.E) {
        if constexpr (sizeof(Pack) >= 4) {
          asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(iwp_tc::smem_u32(slot(i, n))), "l"(from + n * G * VEC),
                       "n"(static_cast<int>(sizeof(Pack)))
                       : "memory");
        } else {  // two bytes are too few for an asynchronous copy
          *slot(i, n) = *reinterpret_cast<const Pack*>(from + n * G * VEC);
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  auto fetch_first = [&] {
#pragma unroll
    for (int i = 0; i < DEPTH - 1; i++) fetch(blockIdx.x + static_cast<int64_t>(i) * gridDim.x, i);
  };

  // ---- counts
  if (alone) {
    cg::cluster_group cluster = cg::this_cluster();
    const int blocks = gridDim.x;
    for (int e = tid; e <= a.E; e += THREADS) sh_mine[e] = 0;
    iwp_tc::launch_next();
    iwp_tc::wait_previous();
    fetch_first();
    __syncthreads();
    const int64_t per = (a.T + blocks - 1) / blocks, t0 = blockIdx.x * per, t1 = min(a.T, t0 + per);
    const int n = __reduce_add_sync(0xFFFFFFFFu, count_ids(a, t0, t1, sh_mine));
    if (lane == 0 && n) atomicAdd(&sh_mine[a.E], n);
    if (blocks > 1)
      cluster.sync();
    else
      __syncthreads();
    for (int e = tid; e <= a.E; e += THREADS) {
      int c = blocks > 1 ? 0 : sh_mine[e];
      if (blocks > 1) {
#pragma unroll
        for (int b = 0; b < MAX_CLUSTER; b++)
          if (b < blocks) c += cluster.map_shared_rank(sh_mine, b)[e];
      }
      sh_count[e] = c;
    }
  } else {
    iwp_tc::launch_next();
    fetch_first();  // inputs: complete before the counting kernel let this one start
    iwp_tc::wait_previous();
    for (int e = tid; e <= a.E; e += THREADS) {
      int c = 0;
#pragma unroll
      for (int b = 0; b < COUNT_PARTS; b++) c += __ldcg(a.part_counts + b * (a.E + 1) + e);
      sh_count[e] = c;
    }
  }
  __syncthreads();
  const int n_tokens = sh_count[a.E];
  const float inv_n = n_tokens > 0 ? 1.f / static_cast<float>(n_tokens) : 0.f;
  const float share = n_tokens > 0 ? 1.f / (static_cast<float>(n_tokens) * static_cast<float>(a.k)) : 0.f;
  const float c = a.coef * static_cast<float>(a.E) * inv_n * a.scale * (a.dloss ? *a.dloss : 1.f);
  for (int e = tid; e < a.E; e += THREADS) {
    sh_f[e] = static_cast<float>(sh_count[e]) * share;
    if (blockIdx.x == 0) a.counts[e] = sh_count[e];
  }
  __syncthreads();

  // ---- rows
  f2 cf[M / 2], sum[M / 2];  // c f_e
#pragma unroll
  for (int i = 0; i < M; i += 2) {
    const int e = (i / VEC * G + g) * VEC + i % VEC, e1 = ((i + 1) / VEC * G + g) * VEC + (i + 1) % VEC;
    cf[i / 2] = pack(e < a.E ? c * sh_f[e] : 0.f, e1 < a.E ? c * sh_f[e1] : 0.f);
    sum[i / 2] = pack(0.f, 0.f);
  }
  constexpr float LOG2E = 1.4426950408889634f;
  const f2 log2e = pack(LOG2E, LOG2E);
  int at = 0;
  for (int64_t step = blockIdx.x; step < steps; step += gridDim.x) {
    const int64_t t = step * rows + tid / G;
    const bool on = ons >> at & 1;
    asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 2) : "memory");
    union {
      Pack p[N];
      E_t x[M];
    } next;
#pragma unroll
    for (int n = 0; n < N; n++) next.p[n] = *slot(at, n);
    fetch(step + (DEPTH - 1) * static_cast<int64_t>(gridDim.x), at == 0 ? DEPTH - 1 : at - 1);
    at = at + 1 == DEPTH ? 0 : at + 1;
    f2 x[M / 2];
    float top = -CUDART_INF_F;
#pragma unroll
    for (int i = 0; i < M; i += 2) {
      const bool in0 = on && (i / VEC * G + g) * VEC < a.E, in1 = on && ((i + 1) / VEC * G + g) * VEC < a.E;
      const float y0 = in0 ? static_cast<float>(next.x[i]) : -CUDART_INF_F, y1 = in1 ? static_cast<float>(next.x[i + 1]) : -CUDART_INF_F;
      top = fmaxf(top, fmaxf(y0, y1));
      x[i / 2] = pack(y0, y1);
    }
    for (int o = G >> 1; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    const float ref = top == -CUDART_INF_F ? 0.f : -top;  // subtracted before the scaling, which lowest values would not survive
    const f2 ref2 = pack(ref, ref);
    f2 s2 = pack(0.f, 0.f), sf2 = s2;
#pragma unroll
    for (int i = 0; i < M / 2; i++) {
      const float2 y = unpack(mul2(add2(x[i], ref2), log2e));
      x[i] = pack(iwp_tc::ex2(y.x), iwp_tc::ex2(y.y));
      s2 = add2(s2, x[i]);
      sf2 = fma2(x[i], cf[i], sf2);
    }
    float s = unpack(s2).x + unpack(s2).y, sf = unpack(sf2).x + unpack(sf2).y;
    for (int o = G >> 1; o; o >>= 1) {
      s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
      sf += __shfl_xor_sync(0xFFFFFFFFu, sf, o);
    }
    const float r = s == 0.f ? 0.f : 1.f / s;  // a row of nothing but -inf (or masked out): p = 0
    const f2 r2 = pack(r, r), minus = pack(-sf * r, -sf * r);
    E_t* const to = static_cast<E_t*>(a.dlogits) + t * a.dlogits_ld + g * VEC;
    const bool write = t < a.T && a.dlogits;
#pragma unroll
    for (int i = 0; i < M / 2; i++) {
      x[i] = mul2(x[i], r2);
      sum[i] = add2(sum[i], x[i]);
      x[i] = mul2(x[i], add2(cf[i], minus));
    }
#pragma unroll
    for (int n = 0; n < N; n++) {
      Pack p;
#pragma unroll
      for (int v = 0; v < VEC; v++) {
        const int i = n * VEC + v;
        const float2 y = unpack(x[i / 2]);
        p.x[v] = static_cast<E_t>(i % 2 ? y.y : y.x);
      }
      if (write && (n * G + g) * VEC < a.E) *reinterpret_cast<Pack*>(to + n * G * VEC) = p;
    }
  }

  // ---- column sums: lanes of a warp, warps of the block, blocks; each in a fixed order
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
  float* const sh_warp = reinterpret_cast<float*>(sh_slots);  // [WARPS][E], at most 32 KB, as E <= 32 M
  static_assert(slot_bytes(M, sizeof(E_t)) >= WARPS * 32 * M * 4 && slot_bytes(M, sizeof(E_t)) >= 4 * MAX_EXPERTS, "room for the sums");
#pragma unroll
  for (int i = 0; i < M; i++) {
    float y = i % 2 ? unpack(sum[i / 2]).y : unpack(sum[i / 2]).x;
    for (int o = G; o < 32; o <<= 1) y += __shfl_xor_sync(0xFFFFFFFFu, y, o);
    const int e = (i / VEC * G + g) * VEC + i % VEC;
    if (lane < G && e < a.E) sh_warp[warp * a.E + e] = y;
  }
  __syncthreads();
  for (int e = tid; e < a.E; e += THREADS) {
    float y = 0.f;
#pragma unroll 8
    for (int w = 0; w < WARPS; w++) y += sh_warp[w * a.E + e];
    sh_sum[e] = y;
    if (!alone) a.part[static_cast<int64_t>(blockIdx.x) * padded(a.E) + e] = y;
  }
  if (alone) {
    cg::cluster_group cluster = cg::this_cluster();
    if (gridDim.x > 1)
      cluster.sync();
    else
      __syncthreads();
    if (blockIdx.x == 0)
      for (int e = tid; e < a.E; e += THREADS) {
        float y = 0.f;
#pragma unroll
        for (int b = 0; b < MAX_CLUSTER; b++)
          if (b < static_cast<int>(gridDim.x)) y += gridDim.x > 1 ? cluster.map_shared_rank(sh_sum, b)[e] : sh_sum[e];
        sh_warp[e] = y;
      }
    if (gridDim.x > 1) cluster.sync();  // nobody leaves while its sums are read
    if (blockIdx.x != 0) return;
    __syncthreads();
  } else {
    __threadfence();
    __syncthreads();
    if (tid == 0) last = atomicInc(&a.hdr->ticket, gridDim.x - 1) == gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    // a thread takes four columns of every groups-th block, then the groups are added in order
    const int quads = padded(a.E) / 4, groups = THREADS / quads;
    if (tid < groups * quads) {
      const int q = tid / quads, e = 4 * (tid - q * quads);
      float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
      for (int b = q; b < static_cast<int>(gridDim.x); b += groups) {
        const float4 z = __ldcg(reinterpret_cast<const float4*>(a.part + static_cast<int64_t>(b) * padded(a.E) + e));
        y.x += z.x, y.y += z.y, y.z += z.z, y.w += z.w;
      }
      *reinterpret_cast<float4*>(sh_warp + q * padded(a.E) + e) = y;
    }
    __syncthreads();
    for (int e = tid; e < a.E; e += THREADS) {
      float y = 0.f;
      for (int i = 0; i < groups; i++) y += sh_warp[i * padded(a.E) + e];
      sh_sum[e] = y;
    }
    __syncthreads();
    for (int e = tid; e < a.E; e += THREADS) sh_warp[e] = sh_sum[e];
    __syncthreads();
  }
  float mine = 0.f;
  for (int e = tid; e < a.E; e += THREADS) {
    const float p = sh_warp[e] * inv_n;
    if (a.mean_prob) a.mean_prob[e] = p;
    mine = fmaf(p, sh_f[e], mine);
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) mine += __shfl_xor_sync(0xFFFFFFFFu, mine, o);
  if (lane == 0) sh_loss[warp] = mine;
  __syncthreads();
  if (tid == 0 && a.loss) {
    float l = 0.f;
    for (int w = 0; w < WARPS; w++) l += sh_loss[w];
    *a.loss = a.coef * static_cast<float>(a.E) * l;
  }
}

}  // namespace iwp_balance
