// iwp_clip.cuh - sums of squares of many tensors in groups, and the tensors times their group's factor.
//
// The tensors are cut into parts of one group each, and a warp takes a part.  Both passes are bound by memory.  Squares are
// added up eight at a time in fp32 and from there on in 64 bits: no sum of gradients that are finite overflows, and
// eights whose squares leave fp32's range are taken in 64 bits from the start.
#pragma once

#include <cooperative_groups.h>

#include "../../include/iwp_clip.h"
#include "iwp_elem.cuh"

namespace iwp_clipper {

using namespace iwp_elem;
namespace cg = cooperative_groups;

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int SMALL_THREADS = 512;  // of the single launch for little work

// rows x cols elements: contiguous if rows == 1.
struct alignas(16) Part {
  const void* in;
  void* out;
  int64_t in_ld, out_ld;
  int rows, cols, group;
  int16_t in_type, out_type;
};
static_assert(sizeof(Part) == 48, "part");

struct Header {
  int status;
  uint32_t ticket;  // wraps to zero with the last block of a launch
};

struct Args {
  Header* hdr;
  const Part* parts;
  const int* first;  // [groups + 1]: the first part of each group
  double* sums;      // [parts]
  double* squares;
  float* norms;
  float* factors;
  int64_t count;  // of parts
  double max_norm, scale;
  int groups, write, have_squares, drop;
};

template <int TYPE>
__device__ __forceinline__ float value(typename Of<TYPE>::T x) {
  return static_cast<float>(x);
}

// Squares of N values, added to a 64-bit sum.
template <int TYPE, int N>
__device__ __forceinline__ void add_squares(const float (&x)[N], double& sum) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < N; i++) s = fmaf(x[i], x[i], s);
  if (TYPE == IWP_F16 || (s >= 0x1p-80f && s <= 0x1.fffffep127f)) {  // (of fp16 values no square leaves fp32's range)
    sum += s;
  } else {
#pragma unroll
    for (int i = 0; i < N; i++) sum = fma(static_cast<double>(x[i]), static_cast<double>(x[i]), sum);
  }
}

// Elements until p is at a multiple of 16 bytes, at most n.
template <int SIZE>
__device__ __forceinline__ int until_aligned(const void* p, int n) {
  const int e = static_cast<int>((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / SIZE;
  return e < n ? e : n;
}

template <int TYPE>
__device__ __forceinline__ void square_run(const void* from, int n, int lane, double& sum) {
  using T = typename Of<TYPE>::T;
  constexpr int VEC = 16 / sizeof(T), WORDS = 8 / VEC, AHEAD = 4;  // eight elements: one or two words
  const T* p = static_cast<const T*>(from);
  const int head = until_aligned<sizeof(T)>(p, n);
  if (lane < head) {
    const float x[1] = {value<TYPE>(p[lane])};
    add_squares<TYPE, 1>(x, sum);
  }
  p += head, n -= head;
  const Word<TYPE, VEC>* const w = reinterpret_cast<const Word<TYPE, VEC>*>(p);
  const int eights = n / 8;
  int i = lane;
  // a warp's lanes read neighbouring words: word u of an eight is 32 further
  for (; i - lane + 32 * AHEAD <= eights; i += 32 * AHEAD) {
    Word<TYPE, VEC> y[AHEAD][WORDS];
#pragma unroll
    for (int a = 0; a < AHEAD; a++)
#pragma unroll
      for (int u = 0; u < WORDS; u++) y[a][u] = w[(i - lane + 32 * a) * WORDS + 32 * u + lane];
#pragma unroll
    for (int a = 0; a < AHEAD; a++) {
      float x[8];
#pragma unroll
      for (int v = 0; v < 8; v++) x[v] = value<TYPE>(y[a][v / VEC].x[v % VEC]);
      add_squares<TYPE, 8>(x, sum);
    }
  }
  for (; i < eights; i += 32) {
    float x[8];
#pragma unroll
    for (int v = 0; v < 8; v++) x[v] = value<TYPE>(w[i * WORDS + v / VEC].x[v % VEC]);
    add_squares<TYPE, 8>(x, sum);
  }
  if (lane < n - eights * 8) {
    const float x[1] = {value<TYPE>(p[eights * 8 + lane])};
    add_squares<TYPE, 1>(x, sum);
  }
}

__device__ __forceinline__ double sum_of(double x) {
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(ALL, x, o);
  return x;
}

template <int TYPE>
__device__ __forceinline__ double square_part(const Part& q, int lane) {
  using T = typename Of<TYPE>::T;
  double sum = 0;
  if (q.rows == 1 || q.cols >= 256) {
    for (int r = 0; r < q.rows; r++) square_run<TYPE>(static_cast<const T*>(q.in) + r * q.in_ld, q.cols, lane, sum);
  } else {
    for (int i = lane; i < q.rows * q.cols; i += 32) {
      const int r = i / q.cols;
      const float x[1] = {value<TYPE>(static_cast<const T*>(q.in)[r * q.in_ld + (i - r * q.cols)])};
      add_squares<TYPE, 1>(x, sum);
    }
  }
  return sum_of(sum);
}

__device__ __forceinline__ double square(const Part& q, int lane) {
  if (q.in_type == IWP_F32) return square_part<IWP_F32>(q, lane);
  if (q.in_type == IWP_BF16) return square_part<IWP_BF16>(q, lane);
  return square_part<IWP_F16>(q, lane);
}

template <int IN, int OUT>
__device__ __forceinline__ typename Of<OUT>::T scaled(typename Of<IN>::T x, float f) {
  return static_cast<typename Of<OUT>::T>(f == 0.f ? 0.f : value<IN>(x) * f);
}

template <int IN, int OUT>
__device__ __forceinline__ void scale_run(const void* from, void* to, int n, int lane, float f) {
  using T = typename Of<IN>::T;
  using U = typename Of<OUT>::T;
  constexpr int VI = 16 / sizeof(T), VO = 16 / sizeof(U), AHEAD = 2;
  constexpr int V = VI > VO ? VI : VO;  // elements a lane takes at a time: whole words of both
  const T* p = static_cast<const T*>(from);
  U* q = static_cast<U*>(to);
  const int head = until_aligned<sizeof(U)>(q, n);
  if (until_aligned<sizeof(T)>(p + head, 1) == 0) {  // both at multiples of 16 bytes from there on
    if (lane < head) q[lane] = scaled<IN, OUT>(p[lane], f);
    p += head, q += head, n -= head;
    const int groups = n / V;
    for (int i = lane; i < groups; i += 32 * AHEAD) {
      Word<IN, VI> x[AHEAD][V / VI];
#pragma unroll
      for (int a = 0; a < AHEAD; a++)
        if (i + 32 * a < groups) {
#pragma unroll
          for (int u = 0; u < V / VI; u++) x[a][u] = reinterpret_cast<const Word<IN, VI>*>(p)[(i + 32 * a) * (V / VI) + u];
        }
#pragma unroll
      for (int a = 0; a < AHEAD; a++)
        if (i + 32 * a < groups) {
#pragma unroll
          for (int u = 0; u < V / VO; u++) {
            Word<OUT, VO> y;
#pragma unroll
            for (int v = 0; v < VO; v++) y.x[v] = scaled<IN, OUT>(x[a][(u * VO + v) / VI].x[(u * VO + v) % VI], f);
            reinterpret_cast<Word<OUT, VO>*>(q)[(i + 32 * a) * (V / VO) + u] = y;
          }
        }
    }
    if (lane < n - groups * V) q[groups * V + lane] = scaled<IN, OUT>(p[groups * V + lane], f);
    return;
  }
  constexpr int SINGLE = 8;
  for (int i = lane; i < n; i += 32 * SINGLE) {
    T x[SINGLE];
#pragma unroll
    for (int a = 0; a < SINGLE; a++)
      if (i + 32 * a < n) x[a] = p[i + 32 * a];
#pragma unroll
    for (int a = 0; a < SINGLE; a++)
      if (i + 32 * a < n) q[i + 32 * a] = scaled<IN, OUT>(x[a], f);
  }
}

template <int IN, int OUT>
__device__ __forceinline__ void scale_part(const Part& q, int lane, float f) {
  using T = typename Of<IN>::T;
  using U = typename Of<OUT>::T;
  if (IN == OUT && q.in == q.out && f == 1.f) return;  // as it is
  if (q.rows == 1 || q.cols >= 256) {
    for (int r = 0; r < q.rows; r++) scale_run<IN, OUT>(static_cast<const T*>(q.in) + r * q.in_ld, static_cast<U*>(q.out) + r * q.out_ld, q.cols, lane, f);
  } else {
    for (int i = lane; i < q.rows * q.cols; i += 32) {
      const int r = i / q.cols, c = i - r * q.cols;
      static_cast<U*>(q.out)[r * q.out_ld + c] = scaled<IN, OUT>(static_cast<const T*>(q.in)[r * q.in_ld + c], f);
    }
  }
}

template <int IN>
__device__ __forceinline__ void scale_from(const Part& q, int lane, float f) {
  if (q.out_type == IWP_F32)
    scale_part<IN, IWP_F32>(q, lane, f);
  else if (q.out_type == IWP_BF16)
    scale_part<IN, IWP_BF16>(q, lane, f);
  else
    scale_part<IN, IWP_F16>(q, lane, f);
}

__device__ __forceinline__ void scale(const Part& q, int lane, float f) {
  if (q.in_type == IWP_F32)
    scale_from<IWP_F32>(q, lane, f);
  else if (q.in_type == IWP_BF16)
    scale_from<IWP_BF16>(q, lane, f);
  else
    scale_from<IWP_F16>(q, lane, f);
}

// A group's sum over its parts, by a warp: lanes take every 32nd part, then the lanes are added.
__device__ __forceinline__ double group_sum(const Args& a, int group, int lane) {
  if (a.have_squares) return a.squares[group];
  double s = 0;
  const int end = a.first[group + 1];
#pragma unroll 8
  for (int i = a.first[group] + lane; i < end; i += 32) s += __ldcg(a.sums + i);
  return sum_of(s);
}

struct Outcome {
  float norm, factor;
};
__device__ __forceinline__ Outcome outcome(const Args& a, double squares) {
  const double norm = sqrt(squares) * fabs(a.scale);
  const bool finite = squares <= 1.7976931348623157e308;  // false for NaN
  double f = a.scale;
  if (!finite)
    f = a.drop ? 0. : f;
  else if (norm > a.max_norm)
    f *= a.max_norm / norm;
  return {static_cast<float>(norm), static_cast<float>(f)};
}

__device__ __forceinline__ void finish_group(const Args& a, int group, double squares) {
  const Outcome o = outcome(a, squares);
  if (!a.have_squares) a.squares[group] = squares;
  a.norms[group] = o.norm;
  if (a.factors) a.factors[group] = o.factor;
}

// Sums, and in the last block to finish the groups' norms and factors.
__global__ void __launch_bounds__(THREADS, 5) k_squares(const Args a) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  launch_next();
  wait_previous();
  const int64_t stride = static_cast<int64_t>(gridDim.x) * WARPS;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * WARPS + warp; i < a.count; i += stride) {
    const double s = square(a.parts[i], lane);
    if (lane == 0) a.sums[i] = s;
  }
  __shared__ bool last;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicInc(&a.hdr->ticket, gridDim.x - 1) == gridDim.x - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  if (a.groups >= WARPS) {
    for (int g = warp; g < a.groups; g += WARPS) {
      const double s = group_sum(a, g, lane);
      if (lane == 0) finish_group(a, g, s);
    }
    return;
  }
  __shared__ double part[WARPS];
  for (int g = 0; g < a.groups; g++) {  // few groups: the whole block sums each
    double s = 0;
    const int end = a.first[g + 1];
#pragma unroll 8
    for (int i = a.first[g] + threadIdx.x; i < end; i += THREADS) s += __ldcg(a.sums + i);
    s = sum_of(s);
    if (lane == 0) part[warp] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
      double y = 0;
      for (int w = 0; w < WARPS; w++) y += part[w];
      finish_group(a, g, y);
    }
    __syncthreads();
  }
}

// Norms and factors from sums that are given.
__global__ void __launch_bounds__(THREADS) k_factors(const Args a) {
  launch_next();
  wait_previous();
  for (int g = blockIdx.x * THREADS + threadIdx.x; g < a.groups; g += gridDim.x * THREADS) finish_group(a, g, a.squares[g]);
}

// Back to front: what the sums read last is still in the L2.
__global__ void __launch_bounds__(THREADS, 4) k_scale(const Args a) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  launch_next();
  wait_previous();
  const int64_t stride = static_cast<int64_t>(gridDim.x) * WARPS;
  for (int64_t i = a.count - 1 - (static_cast<int64_t>(blockIdx.x) * WARPS + warp); i >= 0; i -= stride) {
    const Part& q = a.parts[i];
    scale(q, lane, __ldcg(a.factors + q.group));
  }
}

// All of it in one launch of one cluster, for little work.
__global__ void __launch_bounds__(SMALL_THREADS) k_small(const Args a) {
  const int lane = threadIdx.x & 31, warps = gridDim.x * (SMALL_THREADS / 32);
  const int warp = (threadIdx.x >> 5) * gridDim.x + blockIdx.x;  // neighbouring parts in different CTAs
  cg::cluster_group cluster = cg::this_cluster();
  launch_next();
  wait_previous();
  if (!a.have_squares) {
    for (int64_t i = warp; i < a.count; i += warps) {
      const double s = square(a.parts[i], lane);
      if (lane == 0) __stcg(a.sums + i, s);
    }
    cluster.sync();
  }
  for (int g = warp; g < a.groups; g += warps) {
    const double s = group_sum(a, g, lane);
    if (lane == 0) finish_group(a, g, s);
  }
  if (!a.write) return;
  int group = -1;
  float f = 0.f;
  for (int64_t i = warp; i < a.count; i += warps) {
    const Part& q = a.parts[i];
    if (q.group != group) {
      group = q.group;
      f = outcome(a, group_sum(a, group, lane)).factor;
    }
    scale(q, lane, f);
  }
}

}  // namespace iwp_clipper
