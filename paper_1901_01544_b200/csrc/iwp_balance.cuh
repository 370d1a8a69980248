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
constexpr int COUNT_BLOCKS = 32, COUNT_THREADS = 1024;

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
  int* part_counts;  // [COUNT_BLOCKS][E + 1]: counts, tokens; NULL: the cluster counts for itself
  float* part;       // [gridDim.x][E]
  float* loss;
  float* mean_prob;
  int64_t logits_ld, dlogits_ld, ids_ld, T;
  int E, k, ids_bytes;
  float coef, scale;
};

// Adds the ids of tokens [t0, t1) to a histogram in shared memory (cleared by the caller) and returns this thread's share
// of the number of tokens.
__device__ __forceinline__ int count_ids(const Args& a, int64_t t0, int64_t t1, int* hist) {
  int n = 0;
  for (int64_t i = t0 * a.k + threadIdx.x; i < t1 * a.k; i += blockDim.x) {
    const int64_t t = i / a.k;
    const int j = static_cast<int>(i - t * a.k);
    if (a.mask && !a.mask[t]) continue;
    n += j == 0;
    const int64_t at = t * a.ids_ld + j;
    const int64_t e = a.ids_bytes == 8 ? static_cast<const int64_t*>(a.ids)[at] : static_cast<const int32_t*>(a.ids)[at];
    if (e >= 0 && e < a.E) atomicAdd(&hist[e], 1);
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
  __syncthreads();
  for (int e = threadIdx.x; e <= a.E; e += blockDim.x) a.part_counts[blockIdx.x * (a.E + 1) + e] = hist[e];
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

// Threads of a block, by the number of columns a lane holds (about five registers each).
__host__ __device__ constexpr int threads_of(int columns) { return columns <= 8 ? 1024 : columns <= 16 ? 512 : 256; }

// G lanes share a row; a lane holds N groups of VEC neighbouring columns: columns (n * G + lane) * VEC + v.
template <int TYPE, int VEC, int N>
__global__ void __launch_bounds__(threads_of(VEC* N), 1) k_balance_rows(const Args a, int G) {
  using E_t = typename Elem<TYPE>::T;
  constexpr int THREADS = threads_of(VEC * N), WARPS = THREADS / 32;
  struct alignas(sizeof(E_t) * VEC) Pack {
    E_t x[VEC];
  };
  __shared__ int sh_count[MAX_EXPERTS + 1];
  __shared__ float sh_f[MAX_EXPERTS];
  __shared__ float sh_sum[MAX_EXPERTS];
  __shared__ float sh_warp[8192];  // [WARPS][E]: E <= 32 VEC N, so at most 8192
  __shared__ float sh_loss[32];
  __shared__ bool last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane & (G - 1);
  const bool alone = a.part_counts == nullptr;

  // rows of this block's step s: from (s * gridDim.x + blockIdx.x) * rows on
  const int rows = THREADS / G;
  const int64_t steps = (a.T + rows - 1) / rows;
  Pack next[N];
  bool next_on = false;
  auto fetch = [&](int64_t step) {
    const int64_t t = step * rows + tid / G;
    next_on = step < steps && t < a.T && (!a.mask || a.mask[t]);
#pragma unroll
    for (int n = 0; n < N; n++) {
      const int e = (n * G + g) * VEC;
      if (next_on && e < a.E) next[n] = *reinterpret_cast<const Pack*>(static_cast<const E_t*>(a.logits) + t * a.logits_ld + e);
    }
  };

  // ---- counts
  if (alone) {
    cg::cluster_group cluster = cg::this_cluster();
    const int blocks = gridDim.x;
    for (int e = tid; e <= a.E; e += THREADS) sh_count[e] = 0;
    iwp_tc::launch_next();
    iwp_tc::wait_previous();
    fetch(blockIdx.x);
    __syncthreads();
    const int64_t per = (a.T + blocks - 1) / blocks, t0 = blockIdx.x * per, t1 = min(a.T, t0 + per);
    const int n = __reduce_add_sync(0xFFFFFFFFu, count_ids(a, t0, t1, sh_count));
    if (lane == 0 && n) atomicAdd(&sh_count[a.E], n);
    __syncthreads();
    if (blocks > 1) {
      cluster.sync();
      int total[(MAX_EXPERTS + THREADS) / THREADS];
#pragma unroll
      for (int i = 0; i < (MAX_EXPERTS + THREADS) / THREADS; i++) {
        total[i] = 0;
        const int e = tid + i * THREADS;
        if (e <= a.E)
          for (int b = 0; b < blocks; b++) total[i] += cluster.map_shared_rank(sh_count, b)[e];
      }
      cluster.sync();  // everybody has read everybody's
#pragma unroll
      for (int i = 0; i < (MAX_EXPERTS + THREADS) / THREADS; i++) {
        const int e = tid + i * THREADS;
        if (e <= a.E) sh_count[e] = total[i];
      }
    }
  } else {
    iwp_tc::launch_next();
    fetch(blockIdx.x);  // inputs: complete before the counting kernel let this one start
    iwp_tc::wait_previous();
    for (int e = tid; e <= a.E; e += THREADS) {
      int c = 0;
#pragma unroll 8
      for (int b = 0; b < COUNT_BLOCKS; b++) c += __ldcg(a.part_counts + b * (a.E + 1) + e);
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
  float f[N][VEC], sum[N][VEC];
#pragma unroll
  for (int n = 0; n < N; n++)
#pragma unroll
    for (int v = 0; v < VEC; v++) {
      const int e = (n * G + g) * VEC + v;
      f[n][v] = e < a.E ? sh_f[e] : 0.f;
      sum[n][v] = 0.f;
    }
  for (int64_t step = blockIdx.x; step < steps; step += gridDim.x) {
    const int64_t t = step * rows + tid / G;
    const bool on = next_on;
    float x[N][VEC];
    float top = -CUDART_INF_F;
#pragma unroll
    for (int n = 0; n < N; n++)
#pragma unroll
      for (int v = 0; v < VEC; v++) {
        x[n][v] = on && (n * G + g) * VEC < a.E ? static_cast<float>(next[n].x[v]) : -CUDART_INF_F;
        top = fmaxf(top, x[n][v]);
      }
    fetch(step + gridDim.x);
    for (int o = G >> 1; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    const float ref = top == -CUDART_INF_F ? 0.f : top;
    float s = 0.f, sf = 0.f;
#pragma unroll
    for (int n = 0; n < N; n++)
#pragma unroll
      for (int v = 0; v < VEC; v++) {
        x[n][v] = __expf(x[n][v] - ref);
        s += x[n][v];
        sf = fmaf(x[n][v], f[n][v], sf);
      }
    for (int o = G >> 1; o; o >>= 1) {
      s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
      sf += __shfl_xor_sync(0xFFFFFFFFu, sf, o);
    }
    const float r = s == 0.f ? 0.f : 1.f / s;  // a row of nothing but -inf (or masked out): p = 0
    sf *= r;
#pragma unroll
    for (int n = 0; n < N; n++) {
      const int e = (n * G + g) * VEC;
      Pack p;
#pragma unroll
      for (int v = 0; v < VEC; v++) {
        const float prob = x[n][v] * r;
        sum[n][v] += prob;
        p.x[v] = static_cast<E_t>(on ? c * prob * (f[n][v] - sf) : 0.f);
      }
      if (t < a.T && a.dlogits && e < a.E) *reinterpret_cast<Pack*>(static_cast<E_t*>(a.dlogits) + t * a.dlogits_ld + e) = p;
    }
  }

  // ---- column sums: lanes of a warp, warps of the block, blocks; each in a fixed order
#pragma unroll
  for (int n = 0; n < N; n++)
#pragma unroll
    for (int v = 0; v < VEC; v++) {
      float y = sum[n][v];
      for (int o = G; o < 32; o <<= 1) y += __shfl_xor_sync(0xFFFFFFFFu, y, o);
      const int e = (n * G + g) * VEC + v;
      if (lane < G && e < a.E) sh_warp[warp * a.E + e] = y;
    }
  __syncthreads();
  for (int e = tid; e < a.E; e += THREADS) {
    float y = 0.f;
#pragma unroll 8
    for (int w = 0; w < WARPS; w++) y += sh_warp[w * a.E + e];
    sh_sum[e] = y;
    if (!alone) a.part[static_cast<int64_t>(blockIdx.x) * a.E + e] = y;
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
        for (int b = 0; b < static_cast<int>(gridDim.x); b++) y += gridDim.x > 1 ? cluster.map_shared_rank(sh_sum, b)[e] : sh_sum[e];
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
    // groups of threads take every groups-th block, then the groups are added in order
    const int width = a.E < THREADS ? a.E : THREADS, groups = min(THREADS / width, 8192 / a.E);
    const int q = tid / width;
    if (q < groups)
      for (int e = tid - q * width; e < a.E; e += width) {
        float y = 0.f;
#pragma unroll 8
        for (int b = q; b < static_cast<int>(gridDim.x); b += groups) y += __ldcg(a.part + static_cast<int64_t>(b) * a.E + e);
        sh_warp[q * a.E + e] = y;
      }
    __syncthreads();
    for (int e = tid; e < a.E; e += THREADS) {
      float y = 0.f;
      for (int i = 0; i < groups; i++) y += sh_warp[i * a.E + e];
      sh_sum[e] = y;
    }
    __syncthreads();
    for (int e = tid; e < a.E; e += THREADS) sh_warp[e] = sh_sum[e];
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
