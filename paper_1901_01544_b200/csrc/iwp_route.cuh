// iwp_route.cuh - choice of experts from a router's logits with the weights of the chosen, and the gradient to the logits.
//
// A row of E logits lives in the registers of G lanes (8 up to 256 experts and 8 choices, so that a warp works on four rows at
// a time), M columns per lane, word by word in turn.  A column's key is its choice value in an order-preserving 32-bit code
// whose lowest bits give way to the column's place in its lane.  Every lane sorts its eight largest keys by a network; then the largest
// head is taken k times, ties as the columns go: so they fall to the lower expert.  Of 16-bit logits the codes lose
// nothing.  Where they (or the rounding of scores) may have hidden an order, in a row of a few hundred where values differ, the
// choices in question are put in order by the logits themselves or by scores in 64 bits; a warp makes the row's choice again where even
// that is not enough.  Only the chosen scores have to be exact to the last bits, and only they are computed that way, by k lanes at
// the end.
#pragma once

#include <type_traits>

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
  int64_t logits_ld;
  float weight_scale;
  int T;
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

// Lane g's M columns of a row, in words of VEC that the G lanes take in turn: place i holds column
// ((i / VEC) G + g) VEC + i % VEC.  -inf outside.  (For a type of 16 bits places 2 i and 2 i + 1 are one of `two`.)
template <int TYPE, int M, int G, int VEC>
__device__ __forceinline__ void load_pairs(uint32_t (&two)[M / 2], const typename Of<TYPE>::T* row, int g, int E, bool in) {
  constexpr uint32_t NOTHING = TYPE == IWP_BF16 ? 0xFF80u : 0xFC00u;
#pragma unroll
  for (int n = 0; n < M / VEC; n++) {
    const int first = (n * G + g) * VEC;
    const bool here = in && first < E;
    if constexpr (VEC == 1) {
      uint32_t w = NOTHING;
      if (here) w = *reinterpret_cast<const uint16_t*>(row + first);
      two[n / 2] = n % 2 ? two[n / 2] | w << 16 : w;
    } else {
#pragma unroll
      for (int u = 0; u < VEC / 2; u++) two[n * VEC / 2 + u] = NOTHING << 16 | NOTHING;
      if (here) {
        const Raw<TYPE, VEC> w = *reinterpret_cast<const Raw<TYPE, VEC>*>(row + first);
#pragma unroll
        for (int u = 0; u < VEC / 2; u++) two[n * VEC / 2 + u] = reinterpret_cast<const uint32_t*>(&w)[u];
      }
    }
  }
}
template <int TYPE, int M, int G, int VEC>
__device__ __forceinline__ void load_words(float (&x)[M], const typename Of<TYPE>::T* row, int g, int E, bool in) {
  if constexpr (TYPE != IWP_F32) {
    uint32_t two[M / 2];
    load_pairs<TYPE, M, G, VEC>(two, row, g, E, in);
#pragma unroll
    for (int i = 0; i < M; i++) x[i] = element<TYPE, 2>(two[i / 2], i % 2);
  } else {
#pragma unroll
    for (int n = 0; n < M / VEC; n++) {
      const int first = (n * G + g) * VEC;
#pragma unroll
      for (int v = 0; v < VEC; v++) x[n * VEC + v] = -CUDART_INF_F;
      if (in && first < E) {
        const Raw<TYPE, VEC> w = *reinterpret_cast<const Raw<TYPE, VEC>*>(row + first);
#pragma unroll
        for (int v = 0; v < VEC; v++) x[n * VEC + v] = element<TYPE, VEC>(w, v);
      }
    }
  }
}

// The same columns of results, with `add` added to what is there.
template <int TYPE, int M, int G, int VEC>
__device__ __forceinline__ void store_words(const float (&x)[M], typename Of<TYPE>::T* row, int g, int E, bool add) {
  using T = typename Of<TYPE>::T;
  using W = Word<TYPE, VEC>;
#pragma unroll
  for (int n = 0; n < M / VEC; n++) {
    const int first = (n * G + g) * VEC;
    if (first >= E) continue;
    W w;
    if (add) w = *reinterpret_cast<const W*>(row + first);
#pragma unroll
    for (int v = 0; v < VEC; v++) w.x[v] = static_cast<T>(add ? x[n * VEC + v] + static_cast<float>(w.x[v]) : x[n * VEC + v]);
    *reinterpret_cast<W*>(row + first) = w;
  }
}

// Calls f with the width of a word as a constant.
template <int TYPE, class F>
__device__ __forceinline__ void with_word(int word, const F& f) {
  if constexpr (TYPE != IWP_F32) {
    if (word == 8) return f(std::integral_constant<int, 8>{});
  }
  if (word == 4) return f(std::integral_constant<int, 4>{});
  if (word == 2) return f(std::integral_constant<int, 2>{});
  f(std::integral_constant<int, 1>{});
}

template <int TYPE, int M, int G>
__device__ __forceinline__ void load_columns(float (&x)[M], const typename Of<TYPE>::T* row, int g, int E, bool in, int word) {
  with_word<TYPE>(word, [&](auto v) { load_words<TYPE, M, G, decltype(v)::value>(x, row, g, E, in); });
}

// Two neighbours' arithmetic at once.
template <int TYPE>
struct Pair {
  using T = __nv_bfloat162;
};
template <>
struct Pair<IWP_F16> {
  using T = __half2;
};
template <int TYPE>
__device__ __forceinline__ typename Pair<TYPE>::T pair_of(uint32_t two) {
  return reinterpret_cast<const typename Pair<TYPE>::T&>(two);
}
// Each of two neighbours as 16 bits that order as the values do.
template <int TYPE>
__device__ __forceinline__ uint32_t ordered_pair(uint32_t two) {
  const typename Pair<TYPE>::T zero = pair_of<TYPE>(0), sum = __hadd2_rn(pair_of<TYPE>(two), zero);  // (-0 is 0)
  const uint32_t u = reinterpret_cast<const uint32_t&>(sum);
  uint32_t negative;  // the halves' signs, 16 times each
  asm("prmt.b32 %0, %1, %1, 0xBB99;" : "=r"(negative) : "r"(u));
  return u ^ (negative | 0x80008000u);
}

// Over groups of G lanes.
template <int G>
__device__ __forceinline__ float max_over(float x) {
#pragma unroll
  for (int o = G / 2; o; o /= 2) x = fmaxf(x, __shfl_xor_sync(ALL, x, o));
  return x;
}
template <int G>
__device__ __forceinline__ float sum_over(float x) {
#pragma unroll
  for (int o = G / 2; o; o /= 2) x += __shfl_xor_sync(ALL, x, o);
  return x;
}

// Choice values in fp32 are off: a softmax score by 6 2^-24 of itself and more the further it is from the top (the argument of
// 2^x), which its own size outweighs; and all of a row by a factor from their sum, 52 2^-24 at most (4 + 2 d of each term at
// a distance of d, 5.3 on average at most, and up to 37 additions).  Two of them are then wrong by 64 2^-24 of the largest
// score against each other; the tolerance is 96.  A sigmoid, whose slope falls as its argument's error grows, is off by
// 7 2^-24; the tolerance is 16.  Sums with the bias are rounded by 2^-24 of themselves; the tolerance is twice that.
constexpr float SOFTMAX_TOLERANCE = 0x1.8p-18f, SIGMOID_TOLERANCE = 0x1p-20f;
__device__ __forceinline__ bool apart(float high, float low, float tol) { return high - low > tol + 0x1p-23f * (fabsf(high) + fabsf(low)); }

// As bits that order as the values do, -inf at NONE.
constexpr uint32_t NONE = 0x007FFFFFu;
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);  // (-0 is 0)
  return u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u); }

// Codes that order as the values do, 0 for what is not available.
__device__ __forceinline__ uint64_t code_of(float x) { return x > -CUDART_INF_F ? ordered(x) : 0; }
__device__ __forceinline__ uint64_t code_of(double x) {
  if (!(x > -CUDART_INF)) return 0;
  const uint64_t u = static_cast<uint64_t>(__double_as_longlong(x + 0.));
  return u ^ (static_cast<uint64_t>(static_cast<int64_t>(u) >> 63) | 0x8000000000000000ull);
}
__device__ __forceinline__ double value_of(uint64_t code) {
  return __longlong_as_double(static_cast<int64_t>(code >> 63 ? code ^ 0x8000000000000000ull : ~code));
}
__device__ __forceinline__ uint64_t max_over_warp(uint64_t x) {
  const uint32_t high = __reduce_max_sync(ALL, static_cast<uint32_t>(x >> 32));
  const uint32_t low = __reduce_max_sync(ALL, static_cast<uint32_t>(x >> 32) == high ? static_cast<uint32_t>(x) : 0);
  return static_cast<uint64_t>(high) << 32 | low;
}

// The choice of one row by a whole warp: by the logits, or (SCORES) by scores in 64 bits.  A few rows of a launch come here
// and the launch waits for them, so what there is to do is laid out side by side: 64-bit codes, whose maxima take two
// reductions, and no branches around a column's arithmetic.
template <int TYPE, int M, bool SCORES>
__device__ __noinline__ void choose(const Args& a, int64_t t, int* pick) {
  const int lane = threadIdx.x & 31, size = a.E / a.groups;
  uint64_t code[M];
  {
    float x[M];
    float top = -CUDART_INF_F;
#pragma unroll
    for (int i = 0; i < M; i++) {
      const int e = lane + 32 * i;
      x[i] = e < a.E ? load<TYPE>(a.logits, t * a.logits_ld + e) : -CUDART_INF_F;
      top = fmaxf(top, x[i]);
    }
    if constexpr (SCORES) {
      const bool softmax = a.score == IWP_SOFTMAX;
      top = softmax ? max_over<32>(top) : 0.f;
      if (top == -CUDART_INF_F) top = 0.f;
      double c[M], s = 0;
#pragma unroll
      for (int i = 0; i < M; i++) {
        const double y = softmax ? static_cast<double>(x[i]) - top : -static_cast<double>(x[i]);
        c[i] = exp(y);
        s += c[i];
      }
      if (softmax) {
#pragma unroll
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(ALL, s, o);
      }
#pragma unroll
      for (int i = 0; i < M; i++) {
        const int e = lane + 32 * i;
        double y = (softmax ? c[i] : 1.) / (softmax ? s : 1. + c[i]);
        if (a.bias && e < a.E) y += a.bias[e];
        code[i] = x[i] > -CUDART_INF_F ? code_of(y) : 0;
      }
    } else {
#pragma unroll
      for (int i = 0; i < M; i++) code[i] = code_of(x[i]);
    }
  }
  if (a.groups > 1) {
    uint64_t mine = 0;  // lane q: group q's score
    for (int q = 0; q < a.groups; q++) {
      uint64_t b1 = 0, b2 = 0;
#pragma unroll
      for (int i = 0; i < M; i++) {
        const uint64_t y = (lane + 32 * i) / size == q ? code[i] : 0;
        const uint64_t less = y < b1 ? y : b1;
        b1 = y < b1 ? b1 : y;
        b2 = less < b2 ? b2 : less;
      }
      const uint64_t first = max_over_warp(b1);
      uint64_t score = first;
      if (SCORES && a.group_top == 2) {
        // the second is the largest that is left once one lane has given its first
        const unsigned holders = __ballot_sync(ALL, b1 == first);
        const uint64_t second = max_over_warp(lane == __ffs(holders) - 1 ? b2 : b1);
        score = second ? code_of(value_of(first) + value_of(second)) : 0;
      }
      if (lane == q) mine = score;
    }
    int ahead = 0;
    for (int q = 0; q < a.groups; q++) {
      const uint64_t other = __shfl_sync(ALL, mine, q);
      ahead += other > mine || (other == mine && q < lane);
    }
    const unsigned open = __ballot_sync(ALL, lane < a.groups && ahead < a.top_groups);
#pragma unroll
    for (int i = 0; i < M; i++) {
      const int e = lane + 32 * i;
      if (e < a.E && !(open >> (e / size) & 1)) code[i] = 0;
    }
  }
  if (SCORES && !a.bias) {  // the logits order the scores
#pragma unroll
    for (int i = 0; i < M; i++)
      if (code[i]) code[i] = code_of(load<TYPE>(a.logits, t * a.logits_ld + lane + 32 * i));
  }
  for (int j = 0; j < a.k; j++) {
    uint64_t best = 0;
#pragma unroll
    for (int i = 0; i < M; i++) best = code[i] > best ? code[i] : best;
    const uint64_t m = max_over_warp(best);
    int at = MAX_EXPERTS;
#pragma unroll
    for (int i = M - 1; i >= 0; i--)
      if (code[i] == m) at = lane + 32 * i;
    at = __reduce_min_sync(ALL, at);
#pragma unroll
    for (int i = 0; i < M; i++)
      if (lane + 32 * i == at) code[i] = 0;
    if (lane == 0) pick[j] = m ? at : -1;
  }
}

// A score in 64 bits; sum: of softmax's exponentials below `top`.
static __device__ __noinline__ double exact_score(float x, float top, double sum, bool softmax) {
  const double y = exp(softmax ? static_cast<double>(x) - top : -static_cast<double>(x));
  return softmax ? y / sum : 1. / (1. + y);
}

// The sum of a row's exponentials below `top`, off by 2^-21 of itself at most.  A term is off by two units in the last place of
// expf, 4 2^-24, and by what the rounding of its argument is, half a unit in its last place: 2^-24 from 1 to 2 below the top, 2 2^-24
// from 2 to 4, 4 2^-24 from 4 to 8 and so on.  The further down, the less a term counts: arguments add the most where 1023 of them are 4
// below the top, 0.95 of the sum, and 7.8 2^-24 in all.
template <int TYPE, int M, int G>
__device__ __noinline__ double exact_sum(const typename Of<TYPE>::T* row, int g, int E, bool on, int word, float top) {
  float x[M];
  load_columns<TYPE, M, G>(x, row, g, E, on, word);
  double s = 0;
#pragma unroll
  for (int i = 0; i < M; i++) s += x[i] == -CUDART_INF_F ? 0.f : expf(x[i] - top);
#pragma unroll
  for (int o = G / 2; o; o /= 2) s += __shfl_xor_sync(ALL, s, o);
  return s;
}

// Whether the error of softmax's sum may hide the order of two groups' scores in 64 bits, whose biases follow them: it is common to all
// scores, but not to the biases, so equal sums are so with equal biases alone.  (Two scores of a group are 2 largest at most.)
template <int G>
__device__ __noinline__ bool groups_too_close(const double* score, int groups, int g, float largest) {
  bool close = false;
  for (int q = g; q < groups; q += G)
    for (int p = 0; p < groups; p++) {
      const double mine = score[q], other = score[p];
      if (other > -CUDART_INF && mine > -CUDART_INF && (other != mine || score[groups + p] != score[groups + q]))
        close |= fabs(other - mine) <= 0x1p-20 * largest;
    }
  return close;
}

__device__ __forceinline__ void in_order(uint32_t& a, uint32_t& b) {
  const uint32_t high = max(a, b), low = min(a, b);
  a = high, b = low;
}
// Batcher's odd-even merge sort of eight keys from `first` on, descending.
template <int M>
__device__ __forceinline__ void sort_eight(uint32_t (&x)[M], int first) {
#pragma unroll
  for (int p = 1; p < 8; p *= 2)
#pragma unroll
    for (int k = p; k >= 1; k /= 2)
#pragma unroll
      for (int j = k % p; j <= 7 - k; j += 2 * k)
#pragma unroll
        for (int i = 0; i < k; i++)
          if (i + j + k < 8 && (i + j) / (2 * p) == (i + j + k) / (2 * p)) in_order(x[first + i + j], x[first + i + j + k]);
}
// The eight largest keys, descending, in front: of two sorted eights they are the larger of each pair from opposite ends, which
// are bitonic.
template <int M>
__device__ __forceinline__ void top_eight(uint32_t (&x)[M]) {
  sort_eight(x, 0);
#pragma unroll
  for (int b = 8; b < M; b += 8) {
    sort_eight(x, b);
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] = max(x[i], x[b + 7 - i]);
#pragma unroll
    for (int k = 4; k >= 1; k /= 2)
#pragma unroll
      for (int i = 0; i < 8; i++)
        if (!(i & k)) in_order(x[i], x[i + k]);
  }
}

template <int G>
__device__ __forceinline__ uint32_t key_over(uint32_t x) {
  if constexpr (G == 32) {
    return __reduce_max_sync(ALL, x);
  } else {
#pragma unroll
    for (int o = G / 2; o; o /= 2) x = max(x, __shfl_xor_sync(ALL, x, o));
    return x;
  }
}

// Shared memory of a block of k_route: lanes' sorted keys and a zero behind them (no two of eight lanes share a bank), rows' choices
// (key and lane), counts, a warp's choices made again, and where there are groups a row's keys in the order of the columns and
// the bounds of its groups' scores, or these in 64 bits with the biases in them.
constexpr int WAITING = 12;
struct Shared {
  int waiting, list, hist, pick, row, score, bytes;  // offsets
};
__host__ __device__ inline Shared shared_of(int E, int groups, int G, int M) {
  const int rows = THREADS / G;
  Shared s;
  s.waiting = 0;
  s.list = s.waiting + 4 * THREADS * WAITING;
  s.hist = s.list + 8 * rows * 2 * G;
  s.pick = s.hist + 4 * E;
  s.row = (s.pick + 4 * THREADS + 15) / 16 * 16;
  s.score = s.row + (groups > 1 ? 4 * rows * G * M : 0);
  s.bytes = s.score + (groups > 1 ? 16 * rows * groups : 0);
  return s;
}

__device__ __forceinline__ float reciprocal(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// x = scale x + bias in lane g's columns.
template <int M, int G, int VEC>
__device__ __forceinline__ void add_bias(float (&x)[M], float scale, const float* bias, int g, int E) {
#pragma unroll
  for (int n = 0; n < M / VEC; n++) {
    const int first = (n * G + g) * VEC;
    if (first < E) {
#pragma unroll
      for (int v = 0; v < VEC; v++) x[n * VEC + v] = fmaf(x[n * VEC + v], scale, __ldg(bias + first + v));
    }
  }
}

// Lane g's keys to their columns' places in `keys`.
template <int M, int G, int VEC>
__device__ __forceinline__ void spread_keys(const uint32_t (&key)[M], uint32_t* keys, int g) {
#pragma unroll
  for (int n = 0; n < M / VEC; n++) {
    uint32_t* const to = keys + (n * G + g) * VEC;
    if constexpr (VEC % 4 == 0) {
#pragma unroll
      for (int v = 0; v < VEC; v += 4)
        *reinterpret_cast<uint4*>(to + v) = make_uint4(key[n * VEC + v], key[n * VEC + v + 1], key[n * VEC + v + 2], key[n * VEC + v + 3]);
    } else {
#pragma unroll
      for (int v = 0; v < VEC; v++) to[v] = key[n * VEC + v];
    }
  }
}

// And back.
template <int M, int G, int VEC>
__device__ __forceinline__ void gather_keys(uint32_t (&key)[M], const uint32_t* keys, int g) {
#pragma unroll
  for (int n = 0; n < M / VEC; n++)
#pragma unroll
    for (int v = 0; v < VEC; v++) key[n * VEC + v] = keys[(n * G + g) * VEC + v];
}

// Lane g's keys in groups of `size` columns that are not open become 0.
template <int M, int G, int VEC>
__device__ __forceinline__ void close_groups(uint32_t (&key)[M], unsigned open, int size, int groups, int g) {
  const float per = 1.f / static_cast<float>(size);
  auto is_open = [&](int e) {
    const int q = static_cast<int>((static_cast<float>(e) + 0.5f) * per);  // e / size, exact for e < 1024
    return q >= groups || (open >> q & 1);
  };
#pragma unroll
  for (int n = 0; n < M / VEC; n++) {
    const int first = (n * G + g) * VEC;
    if (size % VEC == 0) {  // a word is of one group
      const bool on = is_open(first);
#pragma unroll
      for (int v = 0; v < VEC; v++) key[n * VEC + v] = on ? key[n * VEC + v] : 0;
    } else {
#pragma unroll
      for (int v = 0; v < VEC; v++) key[n * VEC + v] = is_open(first + v) ? key[n * VEC + v] : 0;
    }
  }
}

// Blocks of k_route that an SM holds, by their registers.
__host__ __device__ constexpr int blocks_of(int M, bool scores) { return M == 8 ? (scores ? 4 : 5) : M == 16 ? 4 : 3; }

// SCORES: the choice goes by scores, or among groups; else by the logits alone.  k <= G: a lane has one pick at most.
// word: elements that all rows are aligned for.
//
// Bound by the integer pipe, which takes a minimum or a maximum every other cycle: 131072 x 256 fp32, 8 choices, 52 us = 2.6 TB/s
// at 260 instructions per row, half of them the sorts'.  (The largest of a lane taken k times from unsorted columns by 32 lanes per
// row: 333 us; sorted, 32 lanes per row: 96.)  bf16 47, with
// sigmoid scores and a bias 67 us; 16384 x 256 bf16, 8 of which 4 groups 18.5 us.  (Left out: lanes that sort four keys 3 us less, but 2 % of
// rows need more of a lane; rows fetched into the L2 ahead 1.5 less, 1 more where rows are short.)
template <int TYPE, int M, int G, bool SCORES>
__global__ void __launch_bounds__(THREADS, blocks_of(M, SCORES)) k_route(const __grid_constant__ Args a, int word) {
  extern __shared__ __align__(16) char smem[];
  using T = typename Of<TYPE>::T;
  constexpr uint32_t LOW = M - 1;  // the bits of a key that hold its place in the lane
  constexpr bool LOSSLESS = !SCORES && TYPE != IWP_F32;  // the type's own 16 bits are in a key
  constexpr uint32_t NO_EXPERT = LOSSLESS && TYPE == IWP_F16 ? 0x03FFFFFFu : NONE;
  constexpr int ROWS = THREADS / G, AGAIN = M * G > 32 ? M * G / 32 : 1;  // columns per lane where a warp has one row
  const Shared at = shared_of(a.E, a.groups, G, M);
  const int tid = threadIdx.x, lane = tid & 31, g = lane & (G - 1), rl = tid / G, row0 = lane & ~(G - 1);
  uint32_t* const waiting = reinterpret_cast<uint32_t*>(smem + at.waiting) + tid * WAITING;
  uint2* const list = reinterpret_cast<uint2*>(smem + at.list) + rl * 2 * G;
  int* const hist = reinterpret_cast<int*>(smem + at.hist);
  int* const pick = reinterpret_cast<int*>(smem + at.pick) + (tid & ~31);
  const unsigned of_row = (G == 32 ? ALL : (1u << G) - 1) << row0, before = ((1u << lane) - 1) & of_row;
  const uint32_t in_word = word - 1;
  const int shift = __popc(in_word);
  auto column = [&](uint32_t place, int of_lane) { return static_cast<int>((((place >> shift) * G + of_lane) << shift) + (place & in_word)); };
  const bool softmax = a.score == IWP_SOFTMAX, renormalize = a.renormalize, count = a.counts != nullptr;
  const bool by_score = SCORES && (a.bias || (a.groups > 1 && a.group_top == 2));
  launch_next();
  for (int e = tid; e < a.E; e += THREADS) hist[e] = 0;
  waiting[8] = 0;
  wait_previous();
  __syncthreads();
  for (int t0 = blockIdx.x * ROWS; t0 < a.T; t0 += gridDim.x * ROWS) {
    const int t = t0 + rl;
    const T* const row = static_cast<const T*>(a.logits) + t * a.logits_ld;
    const bool in = t < a.T, on = in && (!a.mask || a.mask[t]);
    uint32_t key[M];
    bool bad = false;
    uint32_t gone = 0;  // bit i: place i holds a logit of -inf, or no column
    float scale_of_row = 0.f;  // the largest softmax score
    float top = -CUDART_INF_F, s = 0.f, tol = 0.f;  // of the row: largest logit, sum of exponentials below it
    {
      float x[M];
      [[maybe_unused]] uint32_t two[M / 2];
      // rows that hold a NaN or an infinity are looked at again
      bool odd;
      if constexpr (LOSSLESS) {
        with_word<TYPE>(word, [&](auto v) { load_pairs<TYPE, M, G, decltype(v)::value>(two, row, g, a.E, on); });
#pragma unroll
        for (int i = 0; i < M; i++) x[i] = element<TYPE, 2>(two[i / 2], i % 2);
        const auto zero = pair_of<TYPE>(0);
        auto sum = zero;
#pragma unroll
        for (int i = 0; i < M / 2; i++) sum = __hfma2(pair_of<TYPE>(two[i]), zero, sum);
        odd = __hisnan(sum.x) || __hisnan(sum.y);
      } else {
        load_columns<TYPE, M, G>(x, row, g, a.E, on, word);
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < M; i++) sum = fmaf(x[i], 0.f, sum);
        odd = sum != sum;
      }
      if (on && odd) {
#pragma unroll
        for (int i = 0; i < M; i++) {
          bad |= isnan(x[i]) || (softmax && x[i] == CUDART_INF_F);
          if (x[i] == -CUDART_INF_F) gone |= 1u << i;
        }
      }
      bad = (__ballot_sync(ALL, bad) & of_row) != 0;
      if (softmax && (SCORES || !renormalize)) {
#pragma unroll
        for (int i = 0; i < M; i++) top = fmaxf(top, x[i]);
        top = max_over<G>(top);
        if (!renormalize) {
#pragma unroll
          for (int i = 0; i < M; i++) s += x[i] == -CUDART_INF_F ? 0.f : expf(x[i] - top);
          s = sum_over<G>(s);
        }
      }
      if (SCORES && by_score) {
        tol = SIGMOID_TOLERANCE;
        float scale = 1.f;
        if (softmax) {
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < M; i++) {
            x[i] = ex2((x[i] - top) * LOG2E);
            sum += x[i];
          }
          sum = sum_over<G>(sum);
          scale = sum > 0.f ? reciprocal(sum) : 0.f;
          scale_of_row = scale;
          tol = SOFTMAX_TOLERANCE * scale;
        } else {
#pragma unroll
          for (int i = 0; i < M; i++) x[i] = reciprocal(1.f + ex2(-x[i] * LOG2E));
        }
        if (a.bias) {
          with_word<TYPE>(word, [&](auto v) { add_bias<M, G, decltype(v)::value>(x, scale, a.bias, g, a.E); });
        } else {
#pragma unroll
          for (int i = 0; i < M; i++) x[i] *= scale;
        }
#pragma unroll
        for (int i = 0; i < M; i++) key[i] = (ordered(x[i]) & ~LOW) | (LOW - i);
        if (gone) {
#pragma unroll
          for (int i = 0; i < M; i++)
            if (gone >> i & 1) key[i] = 0;
        }
      } else if constexpr (LOSSLESS) {
#pragma unroll
        for (int i = 0; i < M; i += 2) {
          const uint32_t u = ordered_pair<TYPE>(two[i / 2]);
          key[i] = (u << 16) + (LOW - i);
          key[i + 1] = (u & 0xFFFF0000u) | (LOW - i - 1);
        }
      } else {
#pragma unroll
        for (int i = 0; i < M; i++) key[i] = (ordered(x[i]) & ~LOW) | (LOW - i);
      }
    }
    bool again = false;  // by a warp
    if (SCORES && a.groups > 1) {
      const int size = a.E / a.groups;
      uint32_t* const keys = reinterpret_cast<uint32_t*>(smem + at.row) + rl * G * M;
      float* const group_score = reinterpret_cast<float*>(smem + at.score) + rl * 4 * a.groups;  // the least it may be
      float* const group_high = group_score + a.groups;
      with_word<TYPE>(word, [&](auto v) { spread_keys<M, G, decltype(v)::value>(key, keys, g); });
      __syncwarp();
      for (int q = g; q < a.groups; q += G) {
        uint32_t b1 = 0, b2 = 0;
        auto see = [&](uint32_t y) {
          b2 = max(b2, min(b1, y));
          b1 = max(b1, y);
        };
        // (each lane starts at another column, and so at other banks)
        if (size % 4 == 0) {
          int u = q % (size / 4);
#pragma unroll 4
          for (int i = 0; i < size / 4; i++) {
            const uint4 y = *reinterpret_cast<const uint4*>(keys + q * size + 4 * u);
            u = u + 1 == size / 4 ? 0 : u + 1;
            see(y.x), see(y.y), see(y.z), see(y.w);
          }
        } else {
          int u = q % size;
          for (int i = 0; i < size; i++) {
            see(keys[q * size + u]);
            u = u + 1 == size ? 0 : u + 1;
          }
        }
        const bool some = b1 > NONE && (a.group_top == 1 || b2 > NONE);
        float low = -CUDART_INF_F, high = -CUDART_INF_F;
        if (some) {
          low = unordered(b1 & ~LOW), high = unordered(b1 | LOW);
          if (a.group_top == 2) low += unordered(b2 & ~LOW), high += unordered(b2 | LOW);
        }
        group_score[q] = low, group_high[q] = high;
      }
      __syncwarp();
      float least = CUDART_INF_F, most = -CUDART_INF_F;
      unsigned open = 0;  // bit q: group q
      for (int q = g; q < a.groups; q += G) {
        const float mine = group_score[q];
        int ahead = 0;
#pragma unroll 4
        for (int p = 0; p < a.groups; p++) {
          const float other = group_score[p];
          ahead += other > mine || (other == mine && p < q);
        }
        if (ahead < a.top_groups)
          least = fminf(least, mine), open |= 1u << q;
        else
          most = fmaxf(most, group_high[q]);
      }
      least = -max_over<G>(-least);
      most = max_over<G>(most);
#pragma unroll
      for (int o = G / 2; o; o /= 2) open |= __shfl_xor_sync(ALL, open, o);
      const bool question = on && !bad && most > -CUDART_INF_F && least < CUDART_INF_F && !apart(least, most, 2.f * tol);
      if (__any_sync(ALL, question)) {
        // groups' scores in 64 bits, from the columns that make them up
        double* const exact = reinterpret_cast<double*>(group_score);
        const double sum = softmax && by_score ? exact_sum<TYPE, M, G>(row, g, a.E, on, word, top) : 1.;
        __syncwarp();
        for (int q = g; q < a.groups; q += G) {
          uint32_t b1 = 0, b2 = 0, b3 = 0;
          int e1 = 0, e2 = 0;
          for (int e = q * size; e < (q + 1) * size; e++) {
            const uint32_t y = keys[e] | LOW;  // (places do not compare)
            if (y > b1)
              b3 = b2, b2 = b1, e2 = e1, b1 = y, e1 = e;
            else if (y > b2)
              b3 = b2, b2 = y, e2 = e;
            else if (y > b3)
              b3 = y;
          }
          const bool two = a.group_top == 2, some = on && b1 > NONE && (!two || b2 > NONE);
          double score = -CUDART_INF;
          if (some) {
            auto value = [&](int e) {
              const float x = static_cast<float>(row[e]);
              if (!by_score) return static_cast<double>(x);
              const double y = exact_score(x, top, sum, softmax);
              return a.bias ? y + a.bias[e] : y;
            };
            score = value(e1);
            if (two) {
              const double other = value(e2);
              score = score > other ? score + other : other + score;
            }
            // another column may belong in its place, by as little as the codes hide
            const uint32_t in = two ? b2 : b1, out = two ? b3 : b2;
            again |= question && out > NONE && !apart(unordered(in & ~LOW), unordered(out), tol);
          }
          exact[q] = score;
          if (a.bias && some) exact[a.groups + q] = static_cast<double>(a.bias[e1]) + (two ? a.bias[e2] : 0.f);
        }
        __syncwarp();
        if (question) open = 0;
        for (int q = g; q < a.groups; q += G) {
          const double mine = exact[q];
          int ahead = 0;
          for (int p = 0; p < a.groups; p++) {
            const double other = exact[p];
            ahead += other > mine || (other == mine && p < q);
          }
          if (question && ahead < a.top_groups) open |= 1u << q;
        }
        if (softmax && a.bias && question) again |= groups_too_close<G>(exact, a.groups, g, scale_of_row);
#pragma unroll
        for (int o = G / 2; o; o /= 2) open |= __shfl_xor_sync(ALL, open, o);
        again = (__ballot_sync(ALL, again) & of_row) != 0;
        with_word<TYPE>(word, [&](auto v) { gather_keys<M, G, decltype(v)::value>(key, keys, g); });  // (not kept in registers meanwhile)
      }
      with_word<TYPE>(word, [&](auto v) { close_groups<M, G, decltype(v)::value>(key, open, size, a.groups, g); });
      __syncwarp();
    }
    top_eight<M>(key);
    if (SCORES) again |= key[0] > (0xFF800000u | LOW);  // a NaN in the bias
    // the k largest, and one more, to see how far behind it is: a lane's keys wait in shared memory
    reinterpret_cast<uint4*>(waiting)[0] = make_uint4(key[0], key[1], key[2], key[3]);
    reinterpret_cast<uint4*>(waiting)[1] = make_uint4(key[4], key[5], key[6], key[7]);
    uint32_t head = key[0];
    const uint32_t* behind = waiting + 1;
    auto take = [&](int j) {
      // ties: the lower word, then the lower lane (places in a word of different lanes do not compare)
      const bool hit = (head | in_word) == key_over<G>(head | in_word);
      const unsigned holders = __ballot_sync(ALL, hit);
      if (hit && !(holders & before)) {
        list[j] = make_uint2(head, g);
        head = behind == waiting + 9 ? 0 : *behind++;
      }
    };
    int taken = LOSSLESS ? a.k : a.k + 1;
    for (int j = 0; j < taken; j++) take(j);
    __syncwarp();
    auto listed = [&](int j) {  // (key, expert)
      const uint2 p = list[j];
      return make_uint2(p.x, column(LOW - (p.x & LOW), p.y));
    };
    const uint2 mine = listed(g < a.k ? g : 0);
    int e = mine.x > NO_EXPERT && on && g < a.k ? static_cast<int>(mine.y) : -1;
    if (!LOSSLESS) {
      auto close = [&](uint32_t high, uint32_t low) {
        return low > NONE && (SCORES ? !apart(unordered(high & ~LOW), unordered(low | LOW), tol) : (high ^ low) <= LOW);
      };
      const bool question = e >= 0 && !bad && close(mine.x, list[g + 1].x);
      if (__any_sync(ALL, question)) {
        // all that may be as good as the k-th, up to two per lane, in order of what the codes stand for
        auto more = [&] { return on && !bad && close(list[a.k - 1].x, list[taken - 1].x); };
        while (taken < 2 * G && __any_sync(ALL, more())) {
          take(taken++);
          __syncwarp();
        }
        const int n = taken;
        again |= more();
        const bool exact = SCORES && a.bias;
        const double sum = exact && softmax ? exact_sum<TYPE, M, G>(row, g, a.E, on, word, top) : 1.;
        double value[2];
        float bias[2] = {0.f, 0.f};
        int expert[2], rank[2] = {0, 0};
#pragma unroll
        for (int u = 0; u < 2; u++) {
          const int j = g + u * G;
          const uint2 p = listed(j < n ? j : 0);
          const bool there = on && j < n && p.x > NONE;
          expert[u] = there ? static_cast<int>(p.y) : MAX_EXPERTS + j;
          value[u] = -CUDART_INF;
          if (there) {
            const float x = static_cast<float>(row[p.y]);
            if (exact) bias[u] = a.bias[p.y];
            value[u] = exact ? exact_score(x, top, sum, softmax) + bias[u] : static_cast<double>(x);
          }
        }
        for (int i = 0; i < n; i++) {
          const double other = __shfl_sync(ALL, i < G ? value[0] : value[1], row0 + (i & (G - 1)));
          const int its = __shfl_sync(ALL, i < G ? expert[0] : expert[1], row0 + (i & (G - 1)));
#pragma unroll
          for (int u = 0; u < 2; u++) {
            rank[u] += other > value[u] || (other == value[u] && its < expert[u]);
          }
        }
        if (exact && softmax) {
          // the error of softmax's sum is common to all scores, but not to the biases, which may even make values equal that are not
          for (int i = 0; i < n; i++) {
            const double other = __shfl_sync(ALL, i < G ? value[0] : value[1], row0 + (i & (G - 1)));
            const float its_bias = __shfl_sync(ALL, i < G ? bias[0] : bias[1], row0 + (i & (G - 1)));
#pragma unroll
            for (int u = 0; u < 2; u++)
              again |= fabs(other - value[u]) < 0x1p-21 * fabs((other - its_bias) - (value[u] - bias[u]));
          }
        }
        __syncwarp();
#pragma unroll
        for (int u = 0; u < 2; u++)
          if (g + u * G < n && rank[u] < a.k) list[rank[u]].y = expert[u];
        __syncwarp();
        if (e >= 0) e = static_cast<int>(list[g].y);
      }
    }
    float y = e >= 0 ? static_cast<float>(row[e]) : -CUDART_INF_F;
    if (!LOSSLESS || M > 8) {
      // all eight of this lane's keys were taken, and then others: there may have been more here
      if (M > 8 && behind == waiting + 9) again |= list[taken - 1].x != waiting[7] || list[taken - 1].y != g;
      unsigned todo = __ballot_sync(ALL, again && on && !bad);
      while (todo) {
        const int who = __ffs(todo) - 1, who0 = who & ~(G - 1);
        todo &= ~((G == 32 ? ALL : (1u << G) - 1) << who0);
        const int which = __shfl_sync(ALL, t, who);
        if (by_score)
          choose<TYPE, AGAIN, true>(a, which, pick);
        else
          choose<TYPE, AGAIN, false>(a, which, pick);
        __syncwarp();
        if (row0 == who0 && g < a.k) {
          e = pick[g];
          y = e >= 0 ? static_cast<float>(row[e]) : -CUDART_INF_F;
        }
        __syncwarp();
      }
    }
    // weights
    float w = 0.f;
    if (softmax) {
      float ref = top;
      if (renormalize) ref = SCORES ? max_over<G>(y) : __shfl_sync(ALL, y, row0);
      if (y > -CUDART_INF_F) w = expf(y - ref);
    } else {  // sigmoid, times e^-ref, so that scores far below one still have a ratio
      float ref = 0.f;
      if (renormalize) ref = fminf(SCORES ? max_over<G>(y) : __shfl_sync(ALL, y, row0), 0.f);
      if (y > -CUDART_INF_F) {
        const float far = expf(-fabsf(y));
        w = (y >= 0.f ? 1.f : ref == 0.f ? far : expf(y - ref)) / (1.f + far);
      }
    }
    if (renormalize) s = sum_over<G>(w);
    if (softmax || renormalize) w = s > 0.f ? w / s : 0.f;  // (1 if it is the only one)
    w *= a.weight_scale;
    if (bad && on) w = CUDART_NAN_F, e = -1;
    if (in && g < a.k) {
      const int64_t to = static_cast<int64_t>(t) * a.k + g;
      a.weights[to] = w;
      if (a.ids_bytes == 8)
        static_cast<int64_t*>(a.ids)[to] = e;
      else
        static_cast<int32_t*>(a.ids)[to] = e;
      if (count && e >= 0) atomicAdd(&hist[e], 1);
    }
    __syncwarp();  // the list has been read
  }
  if (!count) return;
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
  int64_t logits_ld, ids_ld, weights_ld, dweights_ld, dlogits_ld;
  float inv_scale, scale;
  int T;
  int E, k, score, renormalize, ids_bytes, accumulate;
};

__host__ __device__ constexpr int grad_blocks_of(int M) { return M <= 16 ? 5 : 4; }

// A row's gradient is zero (or, for softmax taken as it is, a multiple of the scores) but at the chosen experts: all of it is
// written in words first, then the chosen ones by a lane each.  Bound by the writes: 131072 x 256 fp32 28 us = 4.8 TB/s, where
// setting the same bytes to zero takes 19 (77 with every lane looking for its columns among
// the chosen).
template <int TYPE, int M, int G>
__global__ void __launch_bounds__(THREADS, grad_blocks_of(M)) k_route_grad(const __grid_constant__ GradArgs a, int word) {
  using T = typename Of<TYPE>::T;
  constexpr int ROWS = THREADS / G;
  const int tid = threadIdx.x, lane = tid & 31, g = lane & (G - 1), rl = tid / G, row0 = lane & ~(G - 1);
  const unsigned of_row = (G == 32 ? ALL : (1u << G) - 1) << row0;
  const bool softmax = a.score == IWP_SOFTMAX, dense = softmax && !a.renormalize;
  launch_next();
  wait_previous();
  // a choice's expert, weight and upstream gradient are fetched a row ahead
  int64_t next_id = -1;
  float next_p = 0.f, next_dw = 0.f;
  auto fetch = [&](int64_t t) {
    next_id = -1;
    if (t < a.T && g < a.k) {
      next_id = load_id(a.ids, a.ids_bytes, t * a.ids_ld + g);
      next_p = a.weights[t * a.weights_ld + g];
      next_dw = a.dweights[t * a.dweights_ld + g];
    }
  };
  fetch(static_cast<int64_t>(blockIdx.x) * ROWS + rl);
  for (int t0 = blockIdx.x * ROWS; t0 < a.T; t0 += gridDim.x * ROWS) {
    const int t = t0 + rl;
    const bool in = t < a.T;
    const T* const row = static_cast<const T*>(a.logits) + t * a.logits_ld;
    T* const out = static_cast<T*>(a.dlogits) + t * a.dlogits_ld;
    const int e = next_id >= 0 && next_id < a.E ? static_cast<int>(next_id) : -1;
    const float p = e >= 0 ? next_p : 0.f, dw = e >= 0 ? next_dw : 0.f;
    fetch(static_cast<int64_t>(t) + static_cast<int64_t>(gridDim.x) * ROWS);
    float y = p * dw;
    const bool some = (__ballot_sync(ALL, e >= 0) & of_row) != 0;
    float x = 0.f, old = 0.f;
    if (e >= 0) {
      if (dense || !softmax) x = static_cast<float>(row[e]);
      if (a.accumulate) old = static_cast<float>(out[e]);
    }
    float v[M];
    if (dense) {
      load_columns<TYPE, M, G>(v, row, g, a.E, in && some, word);
      float top = -CUDART_INF_F, s = 0.f;
#pragma unroll
      for (int i = 0; i < M; i++) top = fmaxf(top, v[i]);
      top = max_over<G>(top);
#pragma unroll
      for (int i = 0; i < M; i++) {
        v[i] = v[i] == -CUDART_INF_F ? 0.f : expf(v[i] - top);
        s += v[i];
      }
      s = sum_over<G>(s);
      const float sum = sum_over<G>(y), f = s > 0.f ? -sum / s : 0.f;
#pragma unroll
      for (int i = 0; i < M; i++) v[i] *= f * a.scale;
      x = x > -CUDART_INF_F ? expf(x - top) * f : 0.f;  // what the chosen expert gets with the others
    } else {
#pragma unroll
      for (int i = 0; i < M; i++) v[i] = 0.f;
      if (a.renormalize) {
        // differences of the upstream gradients, so that nothing is left of a choice of one, and what is left of a sure one is exact
        y = 0.f;
#pragma unroll 4
        for (int i = 0; i < a.k; i++) y = fmaf(__shfl_sync(ALL, p, row0 + i), dw - __shfl_sync(ALL, dw, row0 + i), y);
        y *= p * a.inv_scale;
      }
      if (!softmax) y *= 1.f / (1.f + expf(x));
      x = 0.f;
    }
    // an expert that the row names more than once gets all of it (looked for by shuffles: a match over the lanes takes 2 us more
    // of 131072 x 256)
    bool twice = false;
#pragma unroll 4
    for (int d = 1; d < a.k; d++) twice |= __shfl_sync(ALL, e, row0 + ((g + d) & (G - 1))) == e;
    if (__any_sync(ALL, twice && e >= 0)) {
      float all = 0.f;
#pragma unroll
      for (int i = 0; i < G; i++) {
        const float other = __shfl_sync(ALL, y, row0 + i);
        if (__shfl_sync(ALL, e, row0 + i) == e) all += other;
      }
      y = all;
    }
    __syncwarp();  // what other lanes write has been read
    if (in && (dense || !a.accumulate))
      with_word<TYPE>(word, [&](auto vec) { store_words<TYPE, M, G, decltype(vec)::value>(v, out, g, a.E, a.accumulate); });
    __syncwarp();
    if (e >= 0) out[e] = static_cast<T>(fmaf(y + x, a.scale, old));
  }
}

}  // namespace iwp_router
