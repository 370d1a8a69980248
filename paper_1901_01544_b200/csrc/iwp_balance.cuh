// iwp_balance.cuh - balance loss of a router over E experts: per-expert counts, mean probabilities, loss and gradient.
//
// The gradient of a row needs the counts of the whole batch (f_e) but no other row's probabilities, so the logits are
// read once and the gradient written once: k_balance_counts first (T * top_k ids, a small share of the bytes), then
// k_balance_rows, which keeps a row in the registers of a few lanes: softmax, gradient, and running column sums of p
// for the loss.  The column sums leave each block as one row of partial sums; the last block adds those in order.
// Bound by memory (2 T E elements) for long batches, by the two launches for short ones.
#pragma once

#include <math_constants.h>

#include "../../include/iwp_loss.h"
#include "iwp_tensor.cuh"

namespace iwp_balance {

constexpr int MAX_EXPERTS = 1024;
constexpr int ROW_THREADS = 256;

struct Header {
  int status;
  int n_tokens;
  uint32_t ticket;
  int pad;
};

__global__ void k_balance_counts(Header* hdr, int* counts, const void* ids, int64_t ids_ld, int ids_bytes, const uint8_t* mask, int64_t T,
                                 int k, int E) {
  __shared__ int sh[MAX_EXPERTS];
  __shared__ int sh_n;
  for (int e = threadIdx.x; e < E; e += blockDim.x) sh[e] = 0;
  if (threadIdx.x == 0) sh_n = 0;
  __syncthreads();
  int n = 0;
  for (int64_t i = blockIdx.x * int64_t(blockDim.x) + threadIdx.x; i < T * k; i += int64_t(gridDim.x) * blockDim.x) {
    const int64_t t = i / k;
    const int j = static_cast<int>(i - t * k);
    if (mask && !mask[t]) continue;
    n += j == 0;
    const int64_t at = t * ids_ld + j;
    const int64_t e = ids_bytes == 8 ? static_cast<const int64_t*>(ids)[at] : static_cast<const int32_t*>(ids)[at];
    if (e >= 0 && e < E) atomicAdd(&sh[e], 1);
  }
  if (n) atomicAdd(&sh_n, n);
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += blockDim.x)
    if (sh[e]) atomicAdd(&counts[e], sh[e]);
  if (threadIdx.x == 0 && sh_n) atomicAdd(&hdr->n_tokens, sh_n);
}

struct Rows {
  Header* hdr;
  const int* counts;
  const void* logits;
  const uint8_t* mask;
  const float* dloss;
  void* dlogits;
  float* part;  // [gridDim.x][E]
  float* loss;
  float* mean_prob;
  int64_t logits_ld, dlogits_ld, T;
  int E, k;
  float coef, scale;
};

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

// G lanes share a row; a lane holds N groups of VEC neighbouring columns: columns (n * G + lane) * VEC + v.
template <int TYPE, int VEC, int N>
__global__ void __launch_bounds__(ROW_THREADS) k_balance_rows(const Rows a, int G) {
  using E_t = typename Elem<TYPE>::T;
  struct alignas(sizeof(E_t) * VEC) Pack {
    E_t x[VEC];
  };
  __shared__ float sh_part[MAX_EXPERTS];
  __shared__ float sh_f[MAX_EXPERTS];
  __shared__ bool last;
  const int lane = threadIdx.x & 31, g = lane & (G - 1);
  const int n_tokens = a.hdr->n_tokens;
  const float inv_n = n_tokens > 0 ? 1.f / static_cast<float>(n_tokens) : 0.f;
  const float share = n_tokens > 0 ? 1.f / (static_cast<float>(n_tokens) * static_cast<float>(a.k)) : 0.f;
  const float c = a.coef * static_cast<float>(a.E) * inv_n * a.scale * (a.dloss ? *a.dloss : 1.f);
  for (int e = threadIdx.x; e < a.E; e += blockDim.x) {
    sh_part[e] = 0.f;
    sh_f[e] = static_cast<float>(a.counts[e]) * share;
  }
  __syncthreads();
  float f[N][VEC], sum[N][VEC];
#pragma unroll
  for (int n = 0; n < N; n++)
#pragma unroll
    for (int v = 0; v < VEC; v++) {
      const int e = (n * G + g) * VEC + v;
      f[n][v] = e < a.E ? sh_f[e] : 0.f;
      sum[n][v] = 0.f;
    }
  const int rows_per_block = ROW_THREADS / G;
  const int64_t steps = (a.T + rows_per_block - 1) / rows_per_block;
  for (int64_t step = blockIdx.x; step < steps; step += gridDim.x) {
    const int64_t t = step * rows_per_block + threadIdx.x / G;
    const bool in = t < a.T, on = in && (!a.mask || a.mask[t]);
    float x[N][VEC];
    float top = -CUDART_INF_F;
#pragma unroll
    for (int n = 0; n < N; n++) {
      const int e = (n * G + g) * VEC;
      Pack p;
      const bool here = on && e < a.E;
      if (here) p = *reinterpret_cast<const Pack*>(static_cast<const E_t*>(a.logits) + t * a.logits_ld + e);
#pragma unroll
      for (int v = 0; v < VEC; v++) {
        x[n][v] = here ? static_cast<float>(p.x[v]) : -CUDART_INF_F;
        top = fmaxf(top, x[n][v]);
      }
    }
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
      if (in && a.dlogits && e < a.E) *reinterpret_cast<Pack*>(static_cast<E_t*>(a.dlogits) + t * a.dlogits_ld + e) = p;
    }
  }
  // column sums of the block, warp after warp so that the order is fixed
  for (int w = 0; w < ROW_THREADS / 32; w++) {
    if ((threadIdx.x >> 5) == w) {
#pragma unroll
      for (int n = 0; n < N; n++)
#pragma unroll
        for (int v = 0; v < VEC; v++) {
          float y = sum[n][v];
          for (int o = G; o < 32; o <<= 1) y += __shfl_xor_sync(0xFFFFFFFFu, y, o);
          const int e = (n * G + g) * VEC + v;
          if (lane < G && e < a.E) sh_part[e] += y;
        }
    }
    __syncthreads();
  }
  for (int e = threadIdx.x; e < a.E; e += blockDim.x) a.part[static_cast<int64_t>(blockIdx.x) * a.E + e] = sh_part[e];
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(&a.hdr->ticket, 1u) == gridDim.x - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  float mine = 0.f;
  for (int e = threadIdx.x; e < a.E; e += blockDim.x) {
    float p = 0.f;
#pragma unroll 8
    for (int b = 0; b < static_cast<int>(gridDim.x); b++) p += __ldcg(a.part + static_cast<int64_t>(b) * a.E + e);
    p *= inv_n;
    if (a.mean_prob) a.mean_prob[e] = p;
    mine = fmaf(p, sh_f[e], mine);
  }
  __shared__ float sh_loss[ROW_THREADS / 32];
#pragma unroll
  for (int o = 16; o; o >>= 1) mine += __shfl_xor_sync(0xFFFFFFFFu, mine, o);
  if (lane == 0) sh_loss[threadIdx.x >> 5] = mine;
  __syncthreads();
  if (threadIdx.x == 0) {
    float l = 0.f;
    for (int w = 0; w < ROW_THREADS / 32; w++) l += sh_loss[w];
    if (a.loss) *a.loss = a.coef * static_cast<float>(a.E) * l;
  }
}

}  // namespace iwp_balance
