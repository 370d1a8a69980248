// iwp_clip.cuh - sums of squares of many tensors in groups, and the tensors times their group's factor.
//
// The elements are shared out evenly: a warp has one contiguous range of them, group after group and tensor after tensor, cut
// into parts where tensors, strided rows or the range end.  Both passes are bound by memory.  Squares are added up eight
// at a time in fp32 and from there on in 64 bits: no sum of gradients that are finite overflows, and eights whose squares
// leave fp32's range are taken in 64 bits from the start.
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

// A warp's parts: one here, so that it is there after a single read, and parts [next, end) of the list.
struct alignas(16) Start {
  Part part;
  int next, end;
  int fill[2];
};
static_assert(sizeof(Start) == 64, "start");

struct Header {
  int status;
  uint32_t ticket;  // wraps to zero with the last block of a launch
};

// Warp w leaves its sum over elements of group g at w + g: from one of its groups to the next g grows, and from one warp to
// the next w does, so no two share a place.  A group's sums are at [span.x, span.y).
struct Args {
  Header* hdr;
  const Start* starts;  // [warps]
  const Part* parts;
  const int2* spans;  // [groups]
  double* sums;       // [warps + groups]
  double* squares;
  float* norms;
  float* factors;
  double max_norm, scale;
  int warps, groups, write, have_squares, drop;
  int join;  // k_squares adds up the groups' sums
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

// Elements until p is at a multiple of TO bytes, at most n.
template <int SIZE, int TO = 16>
__device__ __forceinline__ int until_aligned(const void* p, int n) {
  const int e = static_cast<int>((TO - (reinterpret_cast<uintptr_t>(p) & (TO - 1))) & (TO - 1)) / SIZE;
  return e < n ? e : n;
}

template <int TYPE>
__device__ __forceinline__ void square_run(const void* from, int n, int lane, double& sum) {
  using T = typename Of<TYPE>::T;
  constexpr int VEC = 16 / sizeof(T), WORDS = 8 / VEC, AHEAD = 8 / WORDS;  // eight elements: one or two words; eight words in flight
  const T* p = static_cast<const T*>(from);
  const int head = until_aligned<sizeof(T)>(p, n);
  if (lane < head) {
    const float x[1] = {value<TYPE>(p[lane])};
    add_squares<TYPE, 1>(x, sum);
  }
  p += head, n -= head;
  const auto* const w = reinterpret_cast<const Raw<TYPE, VEC>*>(p);
  const int words = n / VEC;
  // a warp's lanes read neighbouring words; word u of a lane's eight is 32 further
  for (int i = lane; i < words; i += 32 * WORDS * AHEAD) {
    Raw<TYPE, VEC> y[AHEAD][WORDS];
#pragma unroll
    for (int a = 0; a < AHEAD; a++)
#pragma unroll
      for (int u = 0; u < WORDS; u++) {
        const int at = i + 32 * (a * WORDS + u);
        y[a][u] = w[at < words ? at : 0];
      }
#pragma unroll
    for (int a = 0; a < AHEAD; a++) {
      float x[8];
#pragma unroll
      for (int v = 0; v < 8; v++) x[v] = i + 32 * (a * WORDS + v / VEC) < words ? element<TYPE, VEC>(y[a][v / VEC], v % VEC) : 0.f;
      if (i + 32 * a * WORDS < words) add_squares<TYPE, 8>(x, sum);
    }
  }
  if (lane < n - words * VEC) {
    const float x[1] = {value<TYPE>(p[words * VEC + lane])};
    add_squares<TYPE, 1>(x, sum);
  }
}

__device__ __forceinline__ double sum_of(double x) {
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(ALL, x, o);
  return x;
}

template <int TYPE>
__device__ __forceinline__ void square_part(const Part& q, int lane, double& sum) {
  using T = typename Of<TYPE>::T;
  if (q.rows == 1 || q.cols >= 256) {
    for (int r = 0; r < q.rows; r++) square_run<TYPE>(static_cast<const T*>(q.in) + r * q.in_ld, q.cols, lane, sum);
  } else {
    for (int i = lane; i < q.rows * q.cols; i += 32) {
      const int r = i / q.cols;
      const float x[1] = {value<TYPE>(static_cast<const T*>(q.in)[r * q.in_ld + (i - r * q.cols)])};
      add_squares<TYPE, 1>(x, sum);
    }
  }
}

__device__ __forceinline__ void square(const Part& q, int lane, double& sum) {
  if (q.in_type == IWP_F32)
    square_part<IWP_F32>(q, lane, sum);
  else if (q.in_type == IWP_BF16)
    square_part<IWP_BF16>(q, lane, sum);
  else
    square_part<IWP_F16>(q, lane, sum);
}

// The product is an fp32 one, and what 16 bits hold is made of that: once in 2^14 values (fp16; bf16 2^17) the first
// rounding brings it to the middle of two of them and so decides.  A multiplication in fp32 and a conversion give the same.
template <int OUT>
__device__ __forceinline__ typename Of<OUT>::T scaled(float x, float f) {
  return static_cast<typename Of<OUT>::T>(f == 0.f ? 0.f : x * f);
}

// The word that starts `by` elements into the first of two neighbouring words.
template <int TYPE, int VEC>
__device__ __forceinline__ Raw<TYPE, VEC> word_between(const Raw<TYPE, VEC>& first, const Raw<TYPE, VEC>& second, int by) {
  constexpr int N = sizeof(Raw<TYPE, VEC>) / 4;
  static_assert(N == 2 || N == 4, "words of 8 or 16 bytes");
  union {
    Raw<TYPE, VEC> two[2];
    uint32_t x[2 * N];
  };
  two[0] = first, two[1] = second;
  const int whole = TYPE == IWP_F32 ? by : by / 2;
#pragma unroll
  for (int i = 0; i < 2 * N - 2; i++) x[i] = N == 4 && (whole & 2) ? x[i + 2] : x[i];
#pragma unroll
  for (int i = 0; i < 2 * N - 1; i++) x[i] = whole & 1 ? x[i + 1] : x[i];
  if constexpr (TYPE != IWP_F32) {
#pragma unroll
    for (int i = 0; i < N; i++) x[i] = by & 1 ? __funnelshift_r(x[i], x[i + 1], 16) : x[i];
  }
  return two[0];
}

// Words of V elements, aligned in `wo`; in `wi` they start `by` elements into a word, and each is made of two.  (25 million bf16
// that are not aligned alike 26 us, aligned ones 23, element by element 35; fp32 into fp32 200 million 392 aligned, 448 made of two,
// 397 element by element.)
template <int IN, int OUT, int V, bool BETWEEN>
__device__ __forceinline__ void scale_words(const Raw<IN, V>* wi, Raw<OUT, V>* wo, int words, int by, int lane, float f) {
  constexpr int AHEAD = BETWEEN ? 2 : 4;
  // back to front, and written past the caches: what the sums read last is read from the L2 again
  for (int i = words ? (words - 1) / (32 * AHEAD) * (32 * AHEAD) + lane : -1; i >= 0; i -= 32 * AHEAD) {
    Raw<IN, V> x[AHEAD], next[AHEAD];
#pragma unroll
    for (int a = 0; a < AHEAD; a++) {
      const int at = min(i + 32 * a, words - 1);
      x[a] = wi[at];
      if constexpr (BETWEEN) next[a] = wi[at + 1];
    }
#pragma unroll
    for (int a = 0; a < AHEAD; a++) {
      if constexpr (BETWEEN) x[a] = word_between<IN, V>(x[a], next[a], by);
      union {
        Word<OUT, V> y;
        Raw<OUT, V> raw;
      };
#pragma unroll
      for (int v = 0; v < V; v++) y.x[v] = scaled<OUT>(element<IN, V>(x[a], v), f);
      if (i + 32 * a < words) __stcs(wo + i + 32 * a, raw);
    }
  }
}

template <int IN, int OUT>
__device__ __forceinline__ void scale_run(const void* from, void* to, int n, int lane, float f) {
  using T = typename Of<IN>::T;
  using U = typename Of<OUT>::T;
  // elements of a lane's word: 16 bytes of the wider type, so that a warp's loads and its stores are both contiguous
  constexpr int V = 16 / (sizeof(T) > sizeof(U) ? sizeof(T) : sizeof(U));
  const T* p = static_cast<const T*>(from);
  U* q = static_cast<U*>(to);
  int head = until_aligned<sizeof(U), V * sizeof(U)>(q, n);
  const int by = static_cast<int>(reinterpret_cast<uintptr_t>(p + head) & (V * sizeof(T) - 1)) / static_cast<int>(sizeof(T));
  if constexpr (sizeof(T) == 4 && sizeof(U) == 4) {
    if (by) {  // one by one: a warp's accesses are whole lines as they are
      constexpr int SINGLE = 8;
      for (int i = lane; i < n; i += 32 * SINGLE) {
        T x[SINGLE];
#pragma unroll
        for (int a = 0; a < SINGLE; a++) x[a] = p[i + 32 * a < n ? i + 32 * a : i];
#pragma unroll
        for (int a = 0; a < SINGLE; a++)
          if (i + 32 * a < n) q[i + 32 * a] = scaled<OUT>(value<IN>(x[a]), f);
      }
      return;
    }
  }
  if (head < by) head = min(head + V, n);  // (no word from before the run, nor from behind it)
  if (lane < head) q[lane] = scaled<OUT>(value<IN>(p[lane]), f);
  p += head, q += head, n -= head;
  const int words = by ? max((n + by) / V - 1, 0) : n / V;
  const auto* const wi = reinterpret_cast<const Raw<IN, V>*>(p - by);
  auto* const wo = reinterpret_cast<Raw<OUT, V>*>(q);
  if constexpr (sizeof(T) == 2 || sizeof(U) == 2)
    if (by) scale_words<IN, OUT, V, true>(wi, wo, words, by, lane, f);
  if (by == 0)
    scale_words<IN, OUT, V, false>(wi, wo, words, by, lane, f);
  if (lane < n - words * V) q[words * V + lane] = scaled<OUT>(value<IN>(p[words * V + lane]), f);
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
      static_cast<U*>(q.out)[r * q.out_ld + c] = scaled<OUT>(value<IN>(static_cast<const T*>(q.in)[r * q.in_ld + c]), f);
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

// A group's sum, by a warp: lanes take every 32nd of the warps' sums, then the lanes are added.
__device__ __forceinline__ double group_sum(const Args& a, int group, int lane) {
  if (a.have_squares) return a.squares[group];
  double s = 0;
  const int2 span = a.spans[group];
#pragma unroll 8
  for (int i = span.x + lane; i < span.y; i += 32) s += __ldcg(a.sums + i);
  return sum_of(s);
}

// The same by a block; the sum is thread 0's.
__device__ __forceinline__ double group_sum_of_block(const Args& a, int group, double (&part)[WARPS]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  double s = 0;
  const int2 span = a.spans[group];
#pragma unroll 16
  for (int i = span.x + threadIdx.x; i < span.y; i += THREADS) s += __ldcg(a.sums + i);
  s = sum_of(s);
  if (lane == 0) part[warp] = s;
  __syncthreads();
  s = 0;
  if (threadIdx.x == 0)
    for (int w = 0; w < WARPS; w++) s += part[w];
  __syncthreads();
  return s;
}

// Sums of warp w's range.
__device__ __forceinline__ void square_range(const Args& a, int w, int lane) {
  const Start start = a.starts[w];
  if (start.end < 0) return;  // nothing left for this warp
  Part q = start.part;
  double sum = 0;
  for (int i = start.next;; i++) {
    const bool more = i < start.end;
    const Part ahead = more ? a.parts[i] : q;
    square(q, lane, sum);
    if (!more || ahead.group != q.group) {
      sum = sum_of(sum);
      if (lane == 0) __stcg(a.sums + w + q.group, sum);
      sum = 0;
    }
    if (!more) return;
    q = ahead;
  }
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

// Squares of eight AlexNet workers (1.95 GB fp32): 287 us = 6.8 TB/s; ResNet-50's 161 tensors: 23 us in fp32 with a norm each,
// 15 in bf16 with one, of which the chain of a block's start, its sum, the ticket and the last block's sum is 5.  (Parts of 16384
// elements dealt out: 359 us, for the last round of them.)
//
// Few groups: the last block to finish adds up the warps' sums (`join`).  Many: a launch of its own, a warp per group.
__global__ void __launch_bounds__(THREADS, 4) k_squares(const Args a) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  wait_previous();
  launch_next();  // after the wait: k_scale may read the table while this kernel runs
  const int w = blockIdx.x * WARPS + warp;
  if (w < a.warps) square_range(a, w, lane);
  if (!a.join) return;
  __shared__ bool last;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicInc(&a.hdr->ticket, gridDim.x - 1) == gridDim.x - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  __shared__ double part[WARPS];
  for (int g = 0; g < a.groups; g++) {
    const double s = group_sum_of_block(a, g, part);
    if (threadIdx.x == 0) finish_group(a, g, s);
  }
}

// A block per group, which a single group of thousands of warps needs, or a warp per group.
template <bool BLOCKS>
__global__ void __launch_bounds__(THREADS) k_groups(const Args a) {
  const int lane = threadIdx.x & 31;
  wait_previous();
  launch_next();
  if constexpr (BLOCKS) {
    __shared__ double part[WARPS];
    for (int g = blockIdx.x; g < a.groups; g += gridDim.x) {
      const double s = a.have_squares ? a.squares[g] : group_sum_of_block(a, g, part);
      if (threadIdx.x == 0) finish_group(a, g, s);
    }
  } else {
    for (int g = blockIdx.x * WARPS + threadIdx.x / 32; g < a.groups; g += gridDim.x * WARPS) {
      const double s = group_sum(a, g, lane);
      if (lane == 0) finish_group(a, g, s);
    }
  }
}

// Each warp its range again.
__device__ __forceinline__ void scale_range(const Args& a, int w, int lane) {
  const Start start = a.starts[w];
  wait_previous();
  int group = -1;
  float f = 0.f;
  for (int i = start.end - 1; i >= start.next - 1; i--) {
    const Part q = i >= start.next ? a.parts[i] : start.part;
    if (q.group != group) group = q.group, f = __ldcg(a.factors + group);
    scale(q, lane, f);
  }
}

// Eight AlexNet workers: 650 us for 3.9 GB = 6.0 TB/s; ResNet-50 bf16 into fp32: 25 us for 153 MB.  (Words of 16 bytes of the
// narrower type, so that a warp's stores left gaps: 69 us.)
__global__ void __launch_bounds__(THREADS, 4) k_scale(const Args a) {
  const int lane = threadIdx.x & 31, w = blockIdx.x * WARPS + threadIdx.x / 32;
  launch_next();
  if (w < a.warps)
    scale_range(a, w, lane);
  else
    wait_previous();
}

// All of it in one launch of one cluster, for little work.
__global__ void __launch_bounds__(SMALL_THREADS) k_small(const Args a) {
  const int lane = threadIdx.x & 31, warps = gridDim.x * (SMALL_THREADS / 32);
  const int warp = (threadIdx.x >> 5) * gridDim.x + blockIdx.x;  // neighbouring ranges in different CTAs
  cg::cluster_group cluster = cg::this_cluster();
  launch_next();
  wait_previous();
  if (!a.have_squares)
    for (int w = warp; w < a.warps; w += warps) square_range(a, w, lane);
  cluster.sync();
  for (int g = warp; g < a.groups; g += warps) {
    const double s = group_sum(a, g, lane);
    if (lane == 0) finish_group(a, g, s);
  }
  if (!a.write) return;
  int group = -1;  // the factors again: no second barrier
  float f = 0.f;
  for (int w = warp; w < a.warps; w += warps) {
    const Start start = a.starts[w];
    for (int i = start.next - 1; i < start.end; i++) {
      const Part q = i >= start.next ? a.parts[i] : start.part;
      if (q.group != group) group = q.group, f = outcome(a, group_sum(a, group, lane)).factor;
      scale(q, lane, f);
    }
  }
}

}  // namespace iwp_clipper
