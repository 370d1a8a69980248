// iwp_route.cuh - choice of experts from a router's logits with the weights of the chosen, and the gradient to the logits.
//
// A row of E logits lives in the registers of G lanes (1 to 32), M neighbouring columns per lane.  The k largest are taken
// one after another: a maximum over the lane's columns, one over the lanes, and the lowest lane and column that hold it (so
// ties go to the lower expert).  Only the chosen scores have to be exact to the last bits, and only they are computed that
// way, by k lanes at the end.
#pragma once

#include "../../include/iwp_route.h"
#include "iwp_elem.cuh"

namespace iwp_router {

using namespace iwp_elem;

constexpr int MAX_EXPERTS = 1024, MAX_TOP = 32, MAX_GROUPS = 32, THREADS = 256;
constexpr float LOG2E = 1.4426950408889634f;

struct State {
  int status;
  uint32_t ticket;  // wraps to zero with the last block of a launch
  int fill[62];
  int counts[MAX_EXPERTS];  // zero between launches
};
static_assert(sizeof(State) == IWP_ROUTE_STATE, "state");

struct Args {
  State* state;
  const void* logits;
  const float* bias;
  const uint8_t* mask;
  void* ids;
  float* weights;
  int* counts;
  int64_t logits_ld, T;
  float weight_scale;
  int E, k, groups, top_groups, group_top, score, renormalize, ids_bytes;
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <int TYPE>
__device__ __forceinline__ float load(const void* p, int64_t at) {
  return static_cast<float>(static_cast<const typename Of<TYPE>::T*>(p)[at]);
}

// M columns from `first` on of a row; -inf outside.
template <int TYPE, int M, int VEC>
__device__ __forceinline__ void load_columns(float (&x)[M], const void* logits, int64_t row, int first, int E, bool in) {
  using W = Word<TYPE, VEC>;
  const auto* p = static_cast<const typename Of<TYPE>::T*>(logits) + row + first;
#pragma unroll
  for (int n = 0; n < M / VEC; n++) {
    if (in && first + n * VEC < E) {
      const W w = *reinterpret_cast<const W*>(p + n * VEC);
#pragma unroll
      for (int v = 0; v < VEC; v++) x[n * VEC + v] = static_cast<float>(w.x[v]);
    } else {
#pragma unroll
      for (int v = 0; v < VEC; v++) x[n * VEC + v] = -CUDART_INF_F;
    }
  }
}

__device__ __forceinline__ float max_over(float x, int G) {
  for (int o = G >> 1; o; o >>= 1) x = fmaxf(x, __shfl_xor_sync(ALL, x, o));
  return x;
}
__device__ __forceinline__ float sum_over(float x, int G) {
  for (int o = G >> 1; o; o >>= 1) x += __shfl_xor_sync(ALL, x, o);
  return x;
}

// The choice of one row in 64 bits, by a whole warp.  Rows come here whose fp32 choice values lie closer than their
// errors, a few in a thousand at most where biases differ.
template <int TYPE>
__device__ __noinline__ void choose_exactly(const Args& a, int64_t t, int* pick) {
  const int lane = threadIdx.x & 31, n = (a.E + 31) / 32;
  double c[MAX_EXPERTS / 32];
  float top = -CUDART_INF_F;
  for (int i = 0; i < n; i++) {
    const int e = lane + 32 * i;
    const float x = e < a.E ? load<TYPE>(a.logits, t * a.logits_ld + e) : -CUDART_INF_F;
    c[i] = x;
    top = fmaxf(top, x);
  }
  top = max_over(top, 32);
  double s = 0;
  if (a.score == IWP_SOFTMAX) {
    for (int i = 0; i < n; i++) {
      if (c[i] > -CUDART_INF) s += exp(c[i] - top);
    }
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(ALL, s, o);
  }
  for (int i = 0; i < n; i++) {
    const int e = lane + 32 * i;
    if (!(c[i] > -CUDART_INF)) continue;
    const double y = a.score == IWP_SOFTMAX ? exp(c[i] - top) / s : 1.0 / (1.0 + exp(-c[i]));
    c[i] = a.bias ? y + a.bias[e] : y;
    if (!(c[i] > -CUDART_INF)) c[i] = -CUDART_INF;
  }
  if (a.groups > 1) {
    const int size = a.E / a.groups;
    double mine = -CUDART_INF;  // lane q: group q's score
    for (int q = 0; q < a.groups; q++) {
      double b1 = -CUDART_INF, b2 = -CUDART_INF;
      for (int i = 0; i < n; i++) {
        const int e = lane + 32 * i;
        if (e / size != q || e >= a.E) continue;
        if (c[i] > b1)
          b2 = b1, b1 = c[i];
        else if (c[i] > b2)
          b2 = c[i];
      }
      for (int o = 16; o; o >>= 1) {
        const double o1 = __shfl_xor_sync(ALL, b1, o), o2 = __shfl_xor_sync(ALL, b2, o);
        b2 = fmax(fmin(b1, o1), fmax(b2, o2));
        b1 = fmax(b1, o1);
      }
      if (lane == q) mine = a.group_top == 2 ? b1 + b2 : b1;
    }
    int ahead = 0;
    for (int q = 0; q < a.groups; q++) {
      const double other = __shfl_sync(ALL, mine, q);
      ahead += other > mine || (other == mine && q < lane);
    }
    const unsigned open = __ballot_sync(ALL, lane < a.groups && ahead < a.top_groups);
    for (int i = 0; i < n; i++) {
      const int e = lane + 32 * i;
      if (e < a.E && !(open >> (e / size) & 1)) c[i] = -CUDART_INF;
    }
  }
  if (!a.bias) {  // the logits order the scores
    for (int i = 0; i < n; i++)
      if (c[i] > -CUDART_INF) c[i] = load<TYPE>(a.logits, t * a.logits_ld + lane + 32 * i);
  }
  for (int j = 0; j < a.k; j++) {
    double m = -CUDART_INF;
    int at = MAX_EXPERTS;
    for (int i = 0; i < n; i++)
      if (c[i] > m) m = c[i], at = lane + 32 * i;
    for (int o = 16; o; o >>= 1) {
      const double om = __shfl_xor_sync(ALL, m, o);
      const int oat = __shfl_xor_sync(ALL, at, o);
      if (om > m || (om == m && oat < at)) m = om, at = oat;
    }
    if (at < MAX_EXPERTS && (at & 31) == lane) c[at / 32] = -CUDART_INF;
    if (lane == 0) pick[j] = at < MAX_EXPERTS ? at : -1;
  }
}

// Shared memory of a block of k_route.
struct Shared {
  int hist, pick, value, row, score, bytes;  // offsets
};
__host__ __device__ inline Shared shared_of(int E, int k, int groups, int G, int M) {
  const int rows = THREADS / G;
  Shared s;
  s.hist = 0;
  s.pick = s.hist + 4 * E;
  s.value = s.pick + 4 * rows * (k + 1);
  s.row = s.value + 4 * rows * k;
  s.score = s.row + (groups > 1 ? 4 * THREADS * M : 0);
  s.bytes = s.score + (groups > 1 ? 4 * rows * groups : 0);
  return s;
}

template <int TYPE, int M, int VEC>
__global__ void __launch_bounds__(THREADS) k_route(const Args a, int G) {
  extern __shared__ __align__(16) char smem[];
  const Shared at = shared_of(a.E, a.k, a.groups, G, M);
  const int tid = threadIdx.x, lane = tid & 31, g = lane & (G - 1), rows = THREADS / G, rl = tid / G;
  int* const hist = reinterpret_cast<int*>(smem + at.hist);
  int* const pick = reinterpret_cast<int*>(smem + at.pick) + rl * (a.k + 1);
  float* const value = reinterpret_cast<float*>(smem + at.value) + rl * a.k;
  float* const row = reinterpret_cast<float*>(smem + at.row) + rl * G * M;
  float* const group_score = reinterpret_cast<float*>(smem + at.score) + rl * a.groups;
  const unsigned of_row = (G == 32 ? ALL : (1u << G) - 1) << (lane & ~(G - 1));
  const int first = g * M;
  const bool softmax = a.score == IWP_SOFTMAX;
  const bool by_score = a.bias || (a.groups > 1 && a.group_top == 2);  // else the logits decide everything
  launch_next();
  for (int e = tid; e < a.E; e += THREADS) hist[e] = 0;
  wait_previous();
  __syncthreads();
  const int64_t steps = (a.T + rows - 1) / rows;
  for (int64_t step = blockIdx.x; step < steps; step += gridDim.x) {
    const int64_t t = step * rows + rl, from = t * a.logits_ld;
    const bool in = t < a.T, on = in && (!a.mask || a.mask[t]);
    float x[M], c[M];
    load_columns<TYPE, M, VEC>(x, a.logits, from, first, a.E, on);
    float top = -CUDART_INF_F;
    bool odd = false;
#pragma unroll
    for (int i = 0; i < M; i++) {
      top = fmaxf(top, x[i]);
      odd |= isnan(x[i]) || (softmax && x[i] == CUDART_INF_F);
    }
    top = max_over(top, G);
    const bool bad = (__ballot_sync(ALL, odd) & of_row) != 0;
    // choice values, and how far two of them may be apart and still be in the wrong order: s is off by at most
    // (2 d + 22) 2^-24 of itself for softmax at a distance of d from the top (2^x, its argument, the sum), so by less than
    // 2^-19 of the largest s; 4 2^-24 for sigmoid, whose slope falls as its argument's error grows
    float tol = 0.f;
    if (by_score) {
      float scale = 1.f;
      if (softmax) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < M; i++) {
          c[i] = x[i] == -CUDART_INF_F ? 0.f : ex2((x[i] - top) * LOG2E);
          s += c[i];
        }
        s = sum_over(s, G);
        scale = s > 0.f ? 1.f / s : 0.f;
      } else {
#pragma unroll
        for (int i = 0; i < M; i++) c[i] = 1.f / (1.f + ex2(-x[i] * LOG2E));
      }
      tol = softmax ? scale * 0x1p-18f : 0x1p-20f;
#pragma unroll
      for (int i = 0; i < M; i++) {
        c[i] *= scale;
        if (a.bias && first + i < a.E) c[i] += a.bias[first + i];
        if (x[i] == -CUDART_INF_F || !(c[i] > -CUDART_INF_F)) c[i] = -CUDART_INF_F;
      }
    } else {
#pragma unroll
      for (int i = 0; i < M; i++) c[i] = x[i];
    }
    bool again = false;  // in 64 bits
    if (a.groups > 1) {
      const int size = a.E / a.groups;
#pragma unroll
      for (int i = 0; i < M; i++) row[first + i] = c[i];
      __syncwarp();
      for (int q = g; q < a.groups; q += G) {
        float b1 = -CUDART_INF_F, b2 = -CUDART_INF_F;
        for (int e = q * size; e < (q + 1) * size; e++) {
          const float y = row[e];
          b2 = fmaxf(b2, fminf(b1, y));
          b1 = fmaxf(b1, y);
        }
        group_score[q] = a.group_top == 2 ? b1 + b2 : b1;
      }
      __syncwarp();
      float least = CUDART_INF_F, most = -CUDART_INF_F;  // of the groups that are open and closed
      unsigned open = 0;                                   // bit n: this lane's n-th group
      for (int q = g, n = 0; q < a.groups; q += G, n++) {
        const float mine = group_score[q];
        int ahead = 0;
        for (int p = 0; p < a.groups; p++) {
          const float other = group_score[p];
          ahead += other > mine || (other == mine && p < q);
        }
        if (ahead < a.top_groups)
          least = fminf(least, mine), open |= 1u << n;
        else
          most = fmaxf(most, mine);
      }
      least = -max_over(-least, G);
      most = max_over(most, G);
      again = by_score && most >= least - (2.f * tol + 0x1p-21f * (fabsf(least) + fabsf(most))) && most > -CUDART_INF_F && least < CUDART_INF_F;
      __syncwarp();
      for (int q = g, n = 0; q < a.groups; q += G, n++) group_score[q] = (open >> n & 1) ? 1.f : 0.f;
      __syncwarp();
#pragma unroll
      for (int i = 0; i < M; i++) {
        if (first + i < a.E && group_score[(first + i) / size] == 0.f) c[i] = -CUDART_INF_F;
        if (!a.bias && c[i] > -CUDART_INF_F) c[i] = x[i];
      }
    }
    // the k largest, and with a bias one more, to see how far behind it is
    const int picks = a.bias ? a.k + 1 : a.k;
    float before = CUDART_INF_F;
    unsigned near = 0;  // bit j: the choice j + 1 is as good as j
    for (int j = 0; j < picks; j++) {
      float best = -CUDART_INF_F;
#pragma unroll
      for (int i = 0; i < M; i++) best = fmaxf(best, c[i]);
      const float m = max_over(best, G);
      const unsigned holders = __ballot_sync(ALL, best == m) & of_row;
      if (lane == __ffs(holders) - 1) {
        int which = -1;
        if (m > -CUDART_INF_F) {
#pragma unroll
          for (int i = 0; i < M; i++)
            if (which < 0 && c[i] == m) which = i, c[i] = -CUDART_INF_F;
        }
        pick[j] = which < 0 ? -1 : first + which;
      }
      if (a.bias && j > 0 && before - m <= tol + 0x1p-21f * (fabsf(before) + fabsf(m))) near |= 1u << (j - 1);
      before = m;
    }
    __syncwarp();
    if (near) {  // equal in logit and bias is equal
      for (int j = 0; j < a.k; j++) {
        if (!(near >> j & 1)) continue;
        const int e0 = pick[j], e1 = pick[j + 1];
        if (e0 < 0 || e1 < 0) continue;
        again |= load<TYPE>(a.logits, from + e0) != load<TYPE>(a.logits, from + e1) || a.bias[e0] != a.bias[e1];
      }
    }
    again = again && on && !bad;
    unsigned todo = __ballot_sync(ALL, again && g == 0);
    while (todo) {
      const int who = __ffs(todo) - 1;
      todo &= todo - 1;
      choose_exactly<TYPE>(a, __shfl_sync(ALL, t, who), reinterpret_cast<int*>(smem + at.pick) + (tid - lane + who) / G * (a.k + 1));
    }
    __syncwarp();
    // weights
    float most = -CUDART_INF_F;
    for (int j = g; j < a.k; j += G) {
      const int e = pick[j];
      const float y = on && e >= 0 ? load<TYPE>(a.logits, from + e) : -CUDART_INF_F;
      value[j] = y;
      most = fmaxf(most, y);
    }
    most = max_over(most, G);
    float s = 0.f;
    if (softmax && !a.renormalize) {
#pragma unroll
      for (int i = 0; i < M; i++) s += x[i] == -CUDART_INF_F ? 0.f : expf(x[i] - top);
    }
    const float ref = softmax ? (a.renormalize ? most : top) : a.renormalize ? fminf(most, 0.f) : 0.f;
    for (int j = g; j < a.k; j += G) {
      const float y = value[j];
      float w = 0.f;
      if (y > -CUDART_INF_F) {
        if (softmax)
          w = expf(y - ref);
        else  // sigmoid, times e^-ref, so that scores far below one still have a ratio
          w = y >= 0.f ? 1.f / (1.f + expf(-y)) : expf(y - ref) / (1.f + expf(y));
      }
      value[j] = w;
      if (a.renormalize) s += w;
    }
    s = sum_over(s, G);
    const float scale = a.renormalize || softmax ? (s > 0.f ? a.weight_scale / s : 0.f) : a.weight_scale;
    for (int j = g; j < a.k; j += G) {
      int e = pick[j];
      if (!on || bad) e = -1;
      const float w = on && bad ? CUDART_NAN_F : e < 0 ? 0.f : value[j] * scale;
      if (in) {
        const int64_t to = t * a.k + j;
        a.weights[to] = w;
        if (a.ids_bytes == 8)
          static_cast<int64_t*>(a.ids)[to] = e;
        else
          static_cast<int32_t*>(a.ids)[to] = e;
        if (a.counts && e >= 0) atomicAdd(&hist[e], 1);
      }
    }
    __syncwarp();
  }
  if (!a.counts) return;
  __syncthreads();
  if (gridDim.x == 1) {
    for (int e = tid; e < a.E; e += THREADS) a.counts[e] = hist[e];
    return;
  }
  // whole numbers: the order of the additions does not matter
  for (int e = tid; e < a.E; e += THREADS)
    if (hist[e]) atomicAdd(&a.state->counts[e], hist[e]);
  __threadfence();
  __shared__ bool last;
  __syncthreads();
  if (tid == 0) last = atomicInc(&a.state->ticket, gridDim.x - 1) == gridDim.x - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  for (int e = tid; e < a.E; e += THREADS) a.counts[e] = atomicExch(&a.state->counts[e], 0);
}

struct GradArgs {
  const void* logits;
  const void* ids;
  const float* weights;
  const float* dweights;
  void* dlogits;
  int64_t logits_ld, ids_ld, weights_ld, dweights_ld, dlogits_ld, T;
  float inv_scale, scale;
  int E, k, score, renormalize, ids_bytes, accumulate;
};

template <int TYPE, int M, int VEC>
__global__ void __launch_bounds__(THREADS) k_route_grad(const GradArgs a, int G) {
  extern __shared__ __align__(16) char smem[];
  using E_t = typename Of<TYPE>::T;
  using W = Word<TYPE, VEC>;
  const int tid = threadIdx.x, lane = tid & 31, g = lane & (G - 1), rows = THREADS / G, rl = tid / G, first = g * M;
  int* const id = reinterpret_cast<int*>(smem) + rl * 2 * a.k;
  float* const value = reinterpret_cast<float*>(id + a.k);
  const unsigned of_row = (G == 32 ? ALL : (1u << G) - 1) << (lane & ~(G - 1));
  const bool softmax = a.score == IWP_SOFTMAX;
  launch_next();
  wait_previous();
  const int64_t steps = (a.T + rows - 1) / rows;
  for (int64_t step = blockIdx.x; step < steps; step += gridDim.x) {
    const int64_t t = step * rows + rl, from = t * a.logits_ld;
    const bool in = t < a.T;
    float v[M];
    float sum = 0.f;
    bool some = false;
    for (int j = g; j < a.k; j += G) {
      const int64_t e = in ? load_id(a.ids, a.ids_bytes, t * a.ids_ld + j) : -1;
      const bool ok = e >= 0 && e < a.E;
      const float y = ok ? a.dweights[t * a.dweights_ld + j] * a.weights[t * a.weights_ld + j] : 0.f;
      id[j] = ok ? static_cast<int>(e) : -1;
      value[j] = y;
      sum += y;
      some |= ok;
    }
    sum = sum_over(sum, G);
    some = (__ballot_sync(ALL, some) & of_row) != 0;
    for (int j = g; j < a.k; j += G) {
      const int e = id[j];
      if (e < 0) continue;
      float y = value[j];
      if (a.renormalize) y -= a.weights[t * a.weights_ld + j] * a.inv_scale * sum;
      if (!softmax) y *= 1.f / (1.f + expf(load<TYPE>(a.logits, from + e)));
      value[j] = y;
    }
    if (softmax && !a.renormalize) {
      load_columns<TYPE, M, VEC>(v, a.logits, from, first, a.E, in && some);
      float top = -CUDART_INF_F, s = 0.f;
#pragma unroll
      for (int i = 0; i < M; i++) top = fmaxf(top, v[i]);
      top = max_over(top, G);
#pragma unroll
      for (int i = 0; i < M; i++) {
        v[i] = v[i] == -CUDART_INF_F ? 0.f : expf(v[i] - top);
        s += v[i];
      }
      s = sum_over(s, G);
      const float f = s > 0.f ? -sum / s : 0.f;
#pragma unroll
      for (int i = 0; i < M; i++) v[i] *= f;
    } else {
#pragma unroll
      for (int i = 0; i < M; i++) v[i] = 0.f;
    }
    __syncwarp();
    for (int j = 0; j < a.k; j++) {
      const int d = id[j] - first;
      const float y = value[j];
      if (id[j] < 0 || d < 0 || d >= M) continue;
#pragma unroll
      for (int i = 0; i < M; i++)
        if (i == d) v[i] += y;
    }
    __syncwarp();
    E_t* const to = static_cast<E_t*>(a.dlogits) + t * a.dlogits_ld + first;
#pragma unroll
    for (int n = 0; n < M / VEC; n++) {
      if (!in || first + n * VEC >= a.E) continue;
      W w;
      if (a.accumulate) {
        w = *reinterpret_cast<const W*>(to + n * VEC);
#pragma unroll
        for (int i = 0; i < VEC; i++) w.x[i] = static_cast<E_t>(fmaf(v[n * VEC + i], a.scale, static_cast<float>(w.x[i])));
      } else {
#pragma unroll
        for (int i = 0; i < VEC; i++) w.x[i] = static_cast<E_t>(v[n * VEC + i] * a.scale);
      }
      *reinterpret_cast<W*>(to + n * VEC) = w;
    }
  }
}

}  // namespace iwp_router
