// iwp_exchange.cuh - slots of (token, expert) pairs in the order of their experts, and rows moved by them.
//
// The order is a counting sort: histograms of contiguous pieces of the pairs, their sums, and ranks within a piece, warp
// by warp in the order of the pairs (so the sort is stable and needs no order of atomics).  Rows are moved in the widest
// words that all rows are aligned for; a token's row is read once for all its experts.
#pragma once

#include "../../include/iwp_route.h"
#include "iwp_elem.cuh"

namespace iwp_exchange {

using namespace iwp_elem;

constexpr int MAX_EXPERTS = 1024, MAX_TOP = 32;
constexpr int ORDER_THREADS = 1024, ORDER_WARPS = ORDER_THREADS / 32;

struct OrderArgs {
  const void* ids;
  int* offsets;
  int* slots;
  int* rows;
  int* part;  // [gridDim.x][E]: pairs of each block; NULL: one block
  int64_t ids_ld;
  int pairs, per_block, E, k, ids_bytes;
};

__device__ __forceinline__ int expert_of(const OrderArgs& a, int p) {
  const int t = p / a.k;
  const int64_t e = load_id(a.ids, a.ids_bytes, t * a.ids_ld + (p - t * a.k));
  return e >= 0 && e < a.E ? static_cast<int>(e) : -1;
}

__global__ void __launch_bounds__(ORDER_THREADS) k_order_count(const OrderArgs a) {
  __shared__ int hist[MAX_EXPERTS];
  const int tid = threadIdx.x;
  launch_next();
  if (tid < a.E) hist[tid] = 0;
  wait_previous();
  __syncthreads();
  const int p0 = blockIdx.x * a.per_block, p1 = min(a.pairs, p0 + a.per_block);
  for (int p = p0 + tid; p < p1; p += ORDER_THREADS) {
    const int e = expert_of(a, p);
    if (e >= 0) atomicAdd(&hist[e], 1);
  }
  __syncthreads();
  if (tid < a.E) a.part[blockIdx.x * a.E + tid] = hist[tid];
}

// Dynamic shared memory: ORDER_WARPS * E counters.
__global__ void __launch_bounds__(ORDER_THREADS) k_order_place(const OrderArgs a) {
  extern __shared__ int count[];  // [warp][E]
  __shared__ int sums[ORDER_WARPS];
  __shared__ int all;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  launch_next();
  for (int i = tid; i < ORDER_WARPS * a.E; i += ORDER_THREADS) count[i] = 0;
  wait_previous();
  __syncthreads();
  // a warp's pairs: a contiguous part of the block's
  const int b0 = blockIdx.x * a.per_block, b1 = min(a.pairs, b0 + a.per_block), per_warp = a.per_block / ORDER_WARPS;
  const int p0 = b0 + warp * per_warp, p1 = min(b1, p0 + per_warp);
  int* const mine = count + warp * a.E;
  for (int p = p0 + lane; p < p1; p += 32) {
    const int e = expert_of(a, p);
    if (e >= 0) atomicAdd(&mine[e], 1);
  }
  __syncthreads();
  int before = 0, total = 0;  // expert tid's pairs in earlier blocks, in all
  if (tid < a.E) {
    if (a.part) {
#pragma unroll 8
      for (int b = 0; b < static_cast<int>(gridDim.x); b++) {
        const int n = __ldcg(a.part + b * a.E + tid);
        total += n;
        if (b < static_cast<int>(blockIdx.x)) before += n;
      }
    } else {
#pragma unroll 8
      for (int w = 0; w < ORDER_WARPS; w++) total += count[w * a.E + tid];
    }
  }
  int upto = total;
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(ALL, upto, o);
    if (lane >= o) upto += y;
  }
  if (lane == 31) sums[warp] = upto;
  __syncthreads();
  for (int w = 0; w < warp; w++) upto += sums[w];
  const int offset = upto - total;
  if (tid == ORDER_THREADS - 1) all = upto;
  if (tid < a.E) {
    int at = offset + before;
#pragma unroll 8
    for (int w = 0; w < ORDER_WARPS; w++) {
      const int n = count[w * a.E + tid];
      count[w * a.E + tid] = at;
      at += n;
    }
    if (blockIdx.x == 0) a.offsets[tid] = offset;
  }
  __syncthreads();
  if (blockIdx.x == 0 && tid == 0) a.offsets[a.E] = all;
  for (int p = p0; p < p1; p += 32) {
    const int e = p + lane < p1 ? expert_of(a, p + lane) : -1;
    const unsigned same = __match_any_sync(ALL, e);
    int slot = -1;
    if (e >= 0) slot = mine[e] + __popc(same & ((1u << lane) - 1));
    __syncwarp();
    if (e >= 0 && lane == __ffs(same) - 1) mine[e] += __popc(same);
    __syncwarp();
    if (p + lane < p1) a.slots[p + lane] = slot;
    if (slot >= 0) a.rows[slot] = (p + lane) / a.k;
  }
  for (int s = all + blockIdx.x * ORDER_THREADS + tid; s < a.pairs; s += gridDim.x * ORDER_THREADS) a.rows[s] = -1;
}

// ---- rows ---------------------------------------------------------------------------------------------

struct RowArgs {
  const int* slots;
  const int* used;  // number of slots that belong to pairs
  const void* by_token;
  const void* by_slot;
  const float* weights;
  void* by_token_out;
  void* by_slot_out;
  float* dweights;
  int64_t by_token_ld, by_slot_ld, weights_ld, by_token_out_ld, by_slot_out_ld;
  int T, D, k;
  int parts;  // a row is shared out to this many warps
};

constexpr int ROW_THREADS = 256, ROW_WARPS = ROW_THREADS / 32;

__device__ __forceinline__ int slot_at(const RowArgs& a, int64_t t, int j) {
  const int s = a.slots[t * a.k + j];
  return s >= 0 && s < a.T * a.k ? s : -1;
}

template <int TYPE, int VEC>
__device__ __forceinline__ void clear_words(typename Of<TYPE>::T* row, int from, int to, int step) {
  Word<TYPE, VEC> zero;
#pragma unroll
  for (int v = 0; v < VEC; v++) zero.x[v] = static_cast<typename Of<TYPE>::T>(0.f);
  for (int i = from; i < to; i += step) reinterpret_cast<Word<TYPE, VEC>*>(row)[i] = zero;
}

// A warp takes part of a token's row to the slots of its pairs.
template <int TYPE, int VEC>
__global__ void __launch_bounds__(ROW_THREADS) k_dispatch(const RowArgs a) {
  using T_t = typename Of<TYPE>::T;
  using W = Word<TYPE, VEC>;
  constexpr int AHEAD = 4;
  const int lane = threadIdx.x & 31, words = a.D / VEC, per = (words + a.parts - 1) / a.parts;
  launch_next();
  wait_previous();
  const int64_t warp = static_cast<int64_t>(blockIdx.x) * ROW_WARPS + threadIdx.x / 32, warps = static_cast<int64_t>(gridDim.x) * ROW_WARPS;
  const int slots = a.T * a.k, used = min(max(*a.used, 0), slots);
  const int64_t items = (static_cast<int64_t>(a.T) + slots - used) * a.parts;
  for (int64_t item = warp; item < items; item += warps) {
    const int64_t t = item / a.parts;
    const int w0 = static_cast<int>(item - t * a.parts) * per, w1 = min(words, w0 + per);
    if (t >= a.T) {
      clear_words<TYPE, VEC>(static_cast<T_t*>(a.by_slot_out) + (used + t - a.T) * a.by_slot_out_ld, w0 + lane, w1, 32);
      continue;
    }
    const W* const from = reinterpret_cast<const W*>(static_cast<const T_t*>(a.by_token) + t * a.by_token_ld);
    int mine = lane < a.k ? slot_at(a, t, lane) : -1;
    for (int w = w0; w < w1; w += 32 * AHEAD) {
      W x[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; u++)
        if (w + 32 * u + lane < w1) x[u] = from[w + 32 * u + lane];
      for (int j = 0; j < a.k; j++) {
        const int s = __shfl_sync(ALL, mine, j);
        if (s < 0) continue;
        W* const to = reinterpret_cast<W*>(static_cast<T_t*>(a.by_slot_out) + s * a.by_slot_out_ld);
#pragma unroll
        for (int u = 0; u < AHEAD; u++)
          if (w + 32 * u + lane < w1) to[w + 32 * u + lane] = x[u];
      }
    }
  }
}

// A warp adds up part of a token's row from the slots of its pairs.
template <int TYPE, int VEC>
__global__ void __launch_bounds__(ROW_THREADS) k_combine(const RowArgs a) {
  using T_t = typename Of<TYPE>::T;
  using W = Word<TYPE, VEC>;
  constexpr int AHEAD = 8;
  const int lane = threadIdx.x & 31, words = a.D / VEC, per = (words + a.parts - 1) / a.parts;
  launch_next();
  wait_previous();
  const int64_t warp = static_cast<int64_t>(blockIdx.x) * ROW_WARPS + threadIdx.x / 32, warps = static_cast<int64_t>(gridDim.x) * ROW_WARPS;
  const int64_t items = static_cast<int64_t>(a.T) * a.parts;
  for (int64_t item = warp; item < items; item += warps) {
    const int64_t t = item / a.parts;
    const int w0 = static_cast<int>(item - t * a.parts) * per, w1 = min(words, w0 + per);
    int mine = lane < a.k ? slot_at(a, t, lane) : -1;
    const float weight = mine < 0 ? 0.f : a.weights ? a.weights[t * a.weights_ld + lane] : 1.f;
    W* const to = reinterpret_cast<W*>(static_cast<T_t*>(a.by_token_out) + t * a.by_token_out_ld);
    for (int w = w0; w < w1; w += 32) {
      const bool in = w + lane < w1;
      float sum[VEC];
#pragma unroll
      for (int v = 0; v < VEC; v++) sum[v] = 0.f;
      for (int j0 = 0; j0 < a.k; j0 += AHEAD) {
        W x[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; u++) {
          const int s = j0 + u < a.k ? __shfl_sync(ALL, mine, j0 + u) : -1;
          if (s >= 0 && in) x[u] = reinterpret_cast<const W*>(static_cast<const T_t*>(a.by_slot) + s * a.by_slot_ld)[w + lane];
        }
#pragma unroll
        for (int u = 0; u < AHEAD; u++) {
          if (j0 + u >= a.k) break;
          const int s = __shfl_sync(ALL, mine, j0 + u);
          const float f = __shfl_sync(ALL, weight, j0 + u);
          if (s < 0) continue;
#pragma unroll
          for (int v = 0; v < VEC; v++) sum[v] = fmaf(f, static_cast<float>(x[u].x[v]), sum[v]);
        }
      }
      if (in) {
        W y;
#pragma unroll
        for (int v = 0; v < VEC; v++) y.x[v] = static_cast<T_t>(sum[v]);
        to[w + lane] = y;
      }
    }
  }
}

// A block takes a token: its row to the slots of its pairs, times their weights, and the products with what the slots hold.
template <int TYPE, int VEC, int K>
__global__ void __launch_bounds__(ROW_THREADS) k_combine_grad(const RowArgs a) {
  using T_t = typename Of<TYPE>::T;
  using W = Word<TYPE, VEC>;
  __shared__ float part[ROW_WARPS][K];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, words = a.D / VEC, threads = blockDim.x;
  launch_next();
  wait_previous();
  const int slots = a.T * a.k, used = min(max(*a.used, 0), slots);
  const int64_t items = static_cast<int64_t>(a.T) + (a.by_slot_out ? slots - used : 0);
  for (int64_t t = blockIdx.x; t < items; t += gridDim.x) {
    if (t >= a.T) {
      clear_words<TYPE, VEC>(static_cast<T_t*>(a.by_slot_out) + (used + t - a.T) * a.by_slot_out_ld, tid, words, threads);
      continue;
    }
    const W* const from = reinterpret_cast<const W*>(static_cast<const T_t*>(a.by_token) + t * a.by_token_ld);
    const int mine = lane < a.k ? slot_at(a, t, lane) : -1;
    const float weight = mine < 0 ? 0.f : a.weights ? a.weights[t * a.weights_ld + lane] : 1.f;
    float dot[K];
#pragma unroll
    for (int j = 0; j < K; j++) dot[j] = 0.f;
    for (int w = 0; w < words; w += threads) {
      const bool in = w + tid < words;
      W dy;
      if (in) dy = from[w + tid];
      for (int j0 = 0; j0 < K; j0 += 8) {
        W x[8];
        if (a.dweights) {
#pragma unroll
          for (int u = 0; u < 8; u++) {
            const int s = __shfl_sync(ALL, mine, j0 + u);
            if (s >= 0 && in) x[u] = reinterpret_cast<const W*>(static_cast<const T_t*>(a.by_slot) + s * a.by_slot_ld)[w + tid];
          }
        }
#pragma unroll
        for (int u = 0; u < 8; u++) {
          const int s = __shfl_sync(ALL, mine, j0 + u);
          const float f = __shfl_sync(ALL, weight, j0 + u);
          if (s < 0 || !in) continue;
          if (a.dweights) {
#pragma unroll
            for (int v = 0; v < VEC; v++) dot[j0 + u] = fmaf(static_cast<float>(dy.x[v]), static_cast<float>(x[u].x[v]), dot[j0 + u]);
          }
          if (a.by_slot_out) {
            W y;
#pragma unroll
            for (int v = 0; v < VEC; v++) y.x[v] = static_cast<T_t>(f * static_cast<float>(dy.x[v]));
            reinterpret_cast<W*>(static_cast<T_t*>(a.by_slot_out) + s * a.by_slot_out_ld)[w + tid] = y;
          }
        }
      }
    }
    if (!a.dweights) continue;
#pragma unroll
    for (int j = 0; j < K; j++) {
      for (int o = 16; o; o >>= 1) dot[j] += __shfl_xor_sync(ALL, dot[j], o);
      if (lane == 0) part[warp][j] = dot[j];
    }
    __syncthreads();
    if (tid < a.k) {
      float y = 0.f;
      for (int w = 0; w < threads / 32; w++) y += part[w][tid];
      a.dweights[t * a.k + tid] = y;
    }
    __syncthreads();
  }
}

}  // namespace iwp_exchange
