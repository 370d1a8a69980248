// iwp_exchange.cuh - slots of (token, expert) pairs in the order of their experts, and rows moved by them.
//
// The order is a counting sort: histograms of contiguous pieces of the pairs, their sums, and ranks within a piece, warp
// by warp in the order of the pairs (so the sort is stable and needs no order of atomics): 131072 pairs of 128 experts in 10 us,
// two launches; 4084 pairs in 7, one block.  Rows are moved in the widest
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

// Dynamic shared memory: ORDER_WARPS * E counters.  A warp keeps up to KEPT * 32 of its pairs' experts in registers.
template <int KEPT>
__global__ void __launch_bounds__(ORDER_THREADS, 1) k_order_place(const OrderArgs a) {
  extern __shared__ int count[];  // [warp][E]
  __shared__ int part[ORDER_THREADS], part_before[ORDER_THREADS];
  __shared__ int sums[ORDER_WARPS];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  launch_next();
  for (int i = tid; i < ORDER_WARPS * a.E; i += ORDER_THREADS) count[i] = 0;
  wait_previous();
  // a warp's pairs: a contiguous part of the block's
  const int b0 = blockIdx.x * a.per_block, b1 = min(a.pairs, b0 + a.per_block), per_warp = a.per_block / ORDER_WARPS;
  const int p0 = b0 + warp * per_warp, p1 = min(b1, p0 + per_warp);
  int* const mine = count + warp * a.E;
  int e[KEPT];
#pragma unroll
  for (int u = 0; u < KEPT; u++) e[u] = p0 + 32 * u + lane < p1 ? expert_of(a, p0 + 32 * u + lane) : -1;
  // expert x's pairs in the blocks before this one, and in all: `groups` threads per expert
  const int groups = ORDER_THREADS / a.E, x = tid % a.E, q = tid / a.E;
  int before = 0, total = 0;
  if (a.part && q < groups) {
#pragma unroll 8
    for (int b = q; b < static_cast<int>(gridDim.x); b += groups) {
      const int n = __ldcg(a.part + b * a.E + x);
      total += n;
      if (b < static_cast<int>(blockIdx.x)) before += n;
    }
    part[tid] = total, part_before[tid] = before;
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < KEPT; u++)
    if (e[u] >= 0) atomicAdd(&mine[e[u]], 1);
  for (int p = p0 + 32 * KEPT + lane; p < p1; p += 32) {
    const int y = expert_of(a, p);
    if (y >= 0) atomicAdd(&mine[y], 1);
  }
  __syncthreads();
  before = total = 0;
  if (tid < a.E) {
    if (a.part) {
      for (int i = 0; i < groups; i++) total += part[i * a.E + tid], before += part_before[i * a.E + tid];
    } else {
#pragma unroll
      for (int w = 0; w < ORDER_WARPS; w++) total += count[w * a.E + tid];
    }
  }
  int upto = total;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(ALL, upto, o);
    if (lane >= o) upto += y;
  }
  if (lane == 31) sums[warp] = upto;
  __syncthreads();
  int ahead = lane < warp ? sums[lane] : 0, all = sums[lane];
#pragma unroll
  for (int o = 16; o; o >>= 1) ahead += __shfl_xor_sync(ALL, ahead, o), all += __shfl_xor_sync(ALL, all, o);
  const int offset = ahead + upto - total;
  if (tid < a.E) {
    int at = offset + before;
#pragma unroll
    for (int w0 = 0; w0 < ORDER_WARPS; w0 += 16) {
      int n[16];
#pragma unroll
      for (int w = 0; w < 16; w++) n[w] = count[(w0 + w) * a.E + tid];
#pragma unroll
      for (int w = 0; w < 16; w++) {
        count[(w0 + w) * a.E + tid] = at;
        at += n[w];
      }
    }
    if (blockIdx.x == 0) a.offsets[tid] = offset;
  }
  if (blockIdx.x == 0 && tid == 0) a.offsets[a.E] = all;
  __syncthreads();
  auto place = [&](int p, int expert) {
    const unsigned same = __match_any_sync(ALL, expert);
    int slot = -1;
    if (expert >= 0) slot = mine[expert] + __popc(same & ((1u << lane) - 1));
    __syncwarp();
    if (expert >= 0 && lane == __ffs(same) - 1) mine[expert] += __popc(same);
    __syncwarp();
    if (p < p1) a.slots[p] = slot;
    if (slot >= 0) a.rows[slot] = p / a.k;
  };
#pragma unroll
  for (int u = 0; u < KEPT; u++)
    if (p0 + 32 * u < p1) place(p0 + 32 * u + lane, e[u]);
  for (int p = p0 + 32 * KEPT; p < p1; p += 32) place(p + lane, p + lane < p1 ? expert_of(a, p + lane) : -1);
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
  int parts;  // a row is shared out to this many warps or blocks
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

// A warp takes part of a token's row to the slots of its pairs.  (16384 x 4096 bf16 to 8 slots each: 206 us = 5.9 TB/s.)
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

// The slots and weights of token t's pairs, by lane; -1 = none.
__device__ __forceinline__ int slots_of(const RowArgs& a, int64_t t, int lane) { return lane < a.k ? slot_at(a, t, lane) : -1; }
__device__ __forceinline__ float weights_of(const RowArgs& a, int64_t t, int lane) {
  return lane >= a.k ? 0.f : a.weights ? a.weights[t * a.weights_ld + lane] : 1.f;
}

constexpr int AT_ONCE = 8;  // rows of slots whose words are in flight together

// A block adds up `blockDim.x` words of a token's row, a word per thread, from the slots of its pairs.
// A row is read by neighbouring warps at the same time, and a row's words stay bits until they are added, in 80 registers:
// 16384 x 4096 bf16 from 8 slots each 184 us = 6.6 TB/s.  (A warp per token, walking along its rows: 569.)
template <int TYPE, int VEC>
__global__ void __launch_bounds__(ROW_THREADS) k_combine(const RowArgs a) {
  using T_t = typename Of<TYPE>::T;
  using W = Word<TYPE, VEC>;
  const int lane = threadIdx.x & 31, words = a.D / VEC;
  launch_next();
  wait_previous();
  const int64_t items = static_cast<int64_t>(a.T) * a.parts;
  int64_t item = blockIdx.x, t = item / a.parts;
  int mine = slots_of(a, t, lane);
  float weight = weights_of(a, t, lane);
  while (item < items) {
    const int word = static_cast<int>(item - t * a.parts) * blockDim.x + threadIdx.x;
    const bool in = word < words;
    // the next token's slots, while this one's rows are read
    const int64_t item2 = item + gridDim.x, t2 = item2 / a.parts;
    const int mine2 = item2 < items ? slots_of(a, t2, lane) : -1;
    const float weight2 = item2 < items ? weights_of(a, t2, lane) : 0.f;
    float sum[VEC];
#pragma unroll
    for (int v = 0; v < VEC; v++) sum[v] = 0.f;
    for (int j0 = 0; j0 < a.k; j0 += AT_ONCE) {
      Raw<TYPE, VEC> x[AT_ONCE];
      unsigned there = 0;
#pragma unroll
      for (int u = 0; u < AT_ONCE; u++) {
        const int s = __shfl_sync(ALL, mine, j0 + u);
        if (s >= 0) there |= 1u << u;
        if (s >= 0 && in) x[u] = reinterpret_cast<const Raw<TYPE, VEC>*>(static_cast<const T_t*>(a.by_slot) + s * a.by_slot_ld)[word];
      }
#pragma unroll
      for (int u = 0; u < AT_ONCE; u++) {
        const float f = __shfl_sync(ALL, weight, j0 + u);
        if (there >> u & 1) {
#pragma unroll
          for (int v = 0; v < VEC; v++) sum[v] = fmaf(f, element<TYPE, VEC>(x[u], v), sum[v]);
        }
      }
    }
    if (in) {
      W y;
#pragma unroll
      for (int v = 0; v < VEC; v++) y.x[v] = static_cast<T_t>(sum[v]);
      reinterpret_cast<W*>(static_cast<T_t*>(a.by_token_out) + t * a.by_token_out_ld)[word] = y;
    }
    item = item2, t = t2, mine = mine2, weight = weight2;
  }
}

// Sums over the lanes of K values each (K a power of two): a lane ends up with one of them, number `sum_of_lane<K>`, the same in
// 32 / K neighbouring lanes.
template <int K>
__device__ __forceinline__ float sums_by_lane(float (&x)[K], int lane) {
  int o = 16;
#pragma unroll
  for (int n = K / 2; n >= 1; n /= 2, o /= 2) {
    const bool up = lane & o;
#pragma unroll
    for (int i = 0; i < n; i++) x[i] = (up ? x[i + n] : x[i]) + __shfl_xor_sync(ALL, up ? x[i] : x[i + n], o);
  }
  for (; o; o /= 2) x[0] += __shfl_xor_sync(ALL, x[0], o);
  return x[0];
}
template <int K>
__device__ __forceinline__ int sum_of_lane(int lane) {
  return lane / (32 / K);
}

// A block takes a token: its row to the slots of its pairs, times their weights, and the products with what the slots hold.
// (16384 x 4096 bf16, 8 slots each, both gradients: 382 us for 2.3 GB = 6.0 TB/s.)
template <int TYPE, int VEC, int K>
__global__ void __launch_bounds__(ROW_THREADS, K == 8 ? 4 : 2) k_combine_grad(const RowArgs a) {
  using T_t = typename Of<TYPE>::T;
  using W = Word<TYPE, VEC>;
  __shared__ float part[2][ROW_WARPS][K];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, words = a.D / VEC, threads = blockDim.x;
  launch_next();
  wait_previous();
  const int slots = a.T * a.k, used = min(max(*a.used, 0), slots);
  int turn = 0;
  int mine = blockIdx.x < a.T ? slots_of(a, blockIdx.x, lane) : -1;
  float weight = blockIdx.x < a.T ? weights_of(a, blockIdx.x, lane) : 0.f;
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
    const auto* const from = reinterpret_cast<const Raw<TYPE, VEC>*>(static_cast<const T_t*>(a.by_token) + t * a.by_token_ld);
    const int64_t t2 = t + gridDim.x;
    const int mine2 = t2 < a.T ? slots_of(a, t2, lane) : -1;
    const float weight2 = t2 < a.T ? weights_of(a, t2, lane) : 0.f;
    float dot[K];
#pragma unroll
    for (int j = 0; j < K; j++) dot[j] = 0.f;
    for (int w = tid; w - tid < words; w += threads) {
      const bool in = w < words;
      Raw<TYPE, VEC> dy;
      if (in) dy = from[w];
#pragma unroll
      for (int j0 = 0; j0 < K; j0 += AT_ONCE) {
        if (j0 >= a.k) break;
        Raw<TYPE, VEC> x[AT_ONCE];
        if (a.dweights) {
#pragma unroll
          for (int u = 0; u < AT_ONCE; u++) {
            const int s = __shfl_sync(ALL, mine, j0 + u);
            if (s >= 0 && in) x[u] = reinterpret_cast<const Raw<TYPE, VEC>*>(static_cast<const T_t*>(a.by_slot) + s * a.by_slot_ld)[w];
          }
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; u++) {
          const int s = __shfl_sync(ALL, mine, j0 + u);
          const float f = __shfl_sync(ALL, weight, j0 + u);
          if (s < 0 || !in) continue;
          if (a.by_slot_out) {
            W y;
#pragma unroll
            for (int v = 0; v < VEC; v++) y.x[v] = static_cast<T_t>(f * element<TYPE, VEC>(dy, v));
            reinterpret_cast<W*>(static_cast<T_t*>(a.by_slot_out) + s * a.by_slot_out_ld)[w] = y;
          }
          if (a.dweights) {
#pragma unroll
            for (int v = 0; v < VEC; v++) dot[j0 + u] = fmaf(element<TYPE, VEC>(dy, v), element<TYPE, VEC>(x[u], v), dot[j0 + u]);
          }
        }
      }
    }
    if (a.dweights) {
      const float sum = sums_by_lane<K>(dot, lane);
      if (lane % (32 / K) == 0) part[turn][warp][sum_of_lane<K>(lane)] = sum;
      __syncthreads();  // (the other half of `part` is read until the next one)
      if (tid < a.k) {
        float y = 0.f;
        for (int w = 0; w < threads / 32; w++) y += part[turn][w][tid];
        a.dweights[t * a.k + tid] = y;
      }
      turn ^= 1;
    }
    mine = mine2, weight = weight2;
  }
  if (a.by_slot_out)
    for (int64_t s = used + blockIdx.x; s < slots; s += gridDim.x)
      clear_words<TYPE, VEC>(static_cast<T_t*>(a.by_slot_out) + s * a.by_slot_out_ld, tid, words, threads);
}

}  // namespace iwp_exchange
