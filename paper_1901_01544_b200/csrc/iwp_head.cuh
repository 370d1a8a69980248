// iwp_head.cuh - output head with its loss (cross entropy, or a teacher's top logits): what happens to the tiles of
// the three products of iwp_tensor.cuh, and the small kernels around them.
//
//   logits pass   z tile -> per row and 32 to 128 columns: maximum and sum of exp (written), the logits at the targets
//                 and, for one piece of the vocabulary, 16-bit codes of how far z is below that maximum
//   rows          per row: lse, loss
//   factors       codes -> row_scale * (exp(z / tau - lse) - q) in the operands' type, in place
//   gradients     dweight = P^T hidden for the piece (complete, since the piece holds every token) and
//                 dhidden = P weight for the piece, summed over the pieces in fp32
//   other pieces  their probabilities come from a second logits product, in the operands' type at once
//
// A vocabulary that fits one piece thus costs three products of 2 T V D operations; of a larger one all but the kept
// piece cost a fourth.  The code of an element costs 4 bytes of traffic, the product it replaces 2 D operations:
// at D = 2048 0.6 against 3 picoseconds.
//
// Cross entropy and distillation differ only in the list of (column, q) that each row subtracts: one entry or top_k
// of them, sorted by column, so that an epilogue warp meets them in the order in which it walks the columns.
#pragma once

#include <math_constants.h>

#include "../../include/iwp_loss.h"
#include "iwp_tensor.cuh"

namespace iwp_head {

using iwp_tc::add2;
using iwp_tc::ex2;
using iwp_tc::f2;
using iwp_tc::fma2;
using iwp_tc::mul2;
using iwp_tc::pack;
using iwp_tc::unpack;
using iwp_tc::Where;

constexpr int MAX_TOP = 1024;
constexpr int NO_COLUMN = 0x7FFFFFFF;
constexpr float LOG2E = 1.4426950408889634f;

// State that outlives a call (and what the kernels of one pass to each other beside it).  The tickets wrap to zero with the last block of each launch.
struct Header {
  int status;
  int n_rows;       // rows with targets
  uint32_t ticket;
  float gmax;       // the largest of the rows' powers of two (k_row_scales)
  int dirty;        // a row that gives nothing has a lse that is not finite; noted while rows are walked
  int clean;        // the same once they all were: dweight reads a copy of the hidden states (clean_rows)
};

// What the rows subtract.  `hard`: one target per row, read as the caller gave them; else lists made by k_soft_targets.
struct Targets {
  const int64_t* hard;
  int64_t ignore;
  int V;
  int k;
  const int* column;       // [T][k] ascending, NO_COLUMN at the end
  const float* q;          // [T][k]
  const float* const_term; // [T] sum of q log q; NaN for a row with an id outside the vocabulary
  const float* scale;      // [T] what the rows' factors are multiplied with, or NULL: 1 for rows with targets

  __device__ __forceinline__ int column_at(int64_t row, int i) const {
    if (!hard) return column[row * k + i];
    const int64_t y = hard[row];
    return y != ignore && y >= 0 && y < V ? static_cast<int>(y) : NO_COLUMN;
  }
  __device__ __forceinline__ float q_at(int64_t row, int i) const { return hard ? 1.f : q[row * k + i]; }
  // the first entry at or after col0, in a list
  __device__ __forceinline__ int first(int64_t row, int col0) const {
    int lo = 0, hi = k;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (column[row * k + mid] < col0)
        lo = mid + 1;
      else
        hi = mid;
    }
    return lo;
  }
  // -1 a target outside the vocabulary, 0 none, 1 some
  __device__ __forceinline__ int state(int64_t row) const {
    if (hard) {
      const int64_t y = hard[row];
      return y == ignore ? 0 : y >= 0 && y < V ? 1 : -1;
    }
    const float c = const_term[row];
    return column[row * k] != NO_COLUMN ? 1 : c != c ? -1 : 0;
  }
  __device__ __forceinline__ float row_scale(int64_t row) const { return state(row) == 1 ? (scale ? scale[row] : 1.f) : 0.f; }
};

// The next targets of a row, in the order of their columns, a few of them fetched ahead.
struct Upcoming {
  int pos, next, after[3];
  __device__ __forceinline__ void none(const Targets& en) {
    pos = en.k;
    next = after[0] = after[1] = after[2] = NO_COLUMN;
  }
  __device__ __forceinline__ void from(const Targets& en, int64_t row, int col0) {
    if (en.hard) {
      none(en);
      const int c = en.column_at(row, 0);
      if (c >= col0 && c != NO_COLUMN) pos = 0, next = c;
      return;
    }
    pos = en.first(row, col0);
    next = pos < en.k ? en.column_at(row, pos) : NO_COLUMN;
#pragma unroll
    for (int i = 0; i < 3; i++) after[i] = pos + 1 + i < en.k ? en.column_at(row, pos + 1 + i) : NO_COLUMN;
  }
  __device__ __forceinline__ void advance(const Targets& en, int64_t row) {
    pos++;
    next = after[0];
    after[0] = after[1];
    after[1] = after[2];
    after[2] = pos + 3 < en.k ? en.column_at(row, pos + 3) : NO_COLUMN;
  }
};

// How the logits pass leaves an element of the kept piece behind in 16 bits, with x = (z - maximum) log2(e) / tau <= 0:
//   bf16 factors: fp16 of 2^(x + 15).  It is the summand at hand anyway, and right to 2^-11 of itself down to 2^-29 of
//     the maximum (0 below 2^-40); the factor is rounded to bf16, eight times as coarse, afterwards.
//   fp16 factors: 16 bits out of the middle of the float y = 8 - x: steps of 2^-12 in log2 above 2^-8 of the maximum, of
//     2^-11 to 2^-24, 0 below.  A probability is right to 8.5e-5 (1.7e-4) of itself, where fp16 of it would be as
//     coarse (2.4e-4 at worst) as the rounding to the factor's type that follows.
enum Codes { NO_CODES = 0, HALF_CODES = 1, LOG_CODES = 2 };
constexpr float SUM_SCALE = 3.0517578125e-5f;  // 2^-15
constexpr float HALF_STEP = 1.220703125e-4f;   // 2^-13: of the finer steps, added before the bits below are cut
constexpr float LOG_END = 31.9998779296875f;   // 32 - 2^-13: the last code, which stands for everything below 2^-24
__device__ __forceinline__ uint32_t log_codes(float y0, float y1) {  // y = 8 - x + HALF_STEP
  y0 = fminf(fmaxf(y0, 8.f), LOG_END);
  y1 = fminf(fmaxf(y1, 8.f), LOG_END);
  return __byte_perm(__float_as_uint(y0), __float_as_uint(y1), 0x6521);
}
// y of a code, in the middle of its step (the coarser steps were cut a quarter of a step off)
__device__ __forceinline__ float log_value(uint32_t code) {
  return code == 0xFFFFu ? CUDART_INF_F : __uint_as_float(((code << 8) + 0x41000000u) | (code >> 15 << 6));
}

// 64 columns of 16 bits of the lane's row (two halves of 16 words) into the warp's next staging area, and from there to the
// matrix of `map` by an asynchronous copy.
__device__ __forceinline__ void copy_out(const CUtensorMap* map, Where& w, const uint32_t (&lo)[16], const uint32_t (&hi)[16], int col0) {
  iwp_tc::staging_free<1>(w.lane);
  char* const area = w.staging + w.area * iwp_tc::STAGING_BYTES;
  w.area ^= 1;
#pragma unroll
  for (int j = 0; j < 4; j++) {
    *reinterpret_cast<uint4*>(iwp_tc::staged(area, w.lane, j)) = make_uint4(lo[4 * j], lo[4 * j + 1], lo[4 * j + 2], lo[4 * j + 3]);
    *reinterpret_cast<uint4*>(iwp_tc::staged(area, w.lane, j + 4)) = make_uint4(hi[4 * j], hi[4 * j + 1], hi[4 * j + 2], hi[4 * j + 3]);
  }
  iwp_tc::store_staged(map, area, w.row0, col0, w.lane);
}

// Column i of the lane's staged row.
__device__ __forceinline__ float* staged_at(const Where& w, int i) {
  return reinterpret_cast<float*>(iwp_tc::staged(w.staging, w.lane, i >> 2)) + (i & 3);
}

// ---- epilogue of the logits pass --------------------------------------------------------------------

template <int CODES>
struct Logits {
  static constexpr bool SUMS = true;
  static constexpr int AREAS = CODES == NO_CODES ? 1 : 2;
  struct Args {
    Targets en;
    int64_t T;
    int V;
    float c;          // log2(e) / tau
    float2* part;     // [T][parts]: maximum of z and sum of 2^((z - maximum) c)
    int parts;
    float* z_at;      // [T][k] logits at the targets
    uint16_t* codes;  // [T][ld] of columns v0 .. v0 + width
    int64_t ld;
    int v0, width;
    CUtensorMap map;  // of the codes, in boxes of 32 rows and 64 columns
  };
  static __device__ __forceinline__ Upcoming begin(const Args& a, const Where& w) {
    Upcoming u;
    u.none(a.en);
    if (w.row0 + w.lane < a.T) u.from(a.en, w.row0 + w.lane, w.col0);
    return u;
  }
  static __device__ __forceinline__ void tile(const Args& a, Where& w, Upcoming& up, f2 (&acc)[iwp_tc::TILE_N / 4]) {
    constexpr int CHUNKS = iwp_tc::TILE_N / 64;
    const int row = w.row0 + w.lane;
    const bool live = row < a.T;
    float top = -CUDART_INF_F;
#pragma unroll
    for (int c = 0; c < CHUNKS; c++) {
      const int c0 = w.col0 + 32 * c;
      if (32 * c >= w.width) break;
      if (__any_sync(0xFFFFFFFFu, up.next < c0 + 32)) {  // some row has a target here
        iwp_tc::staging_free<0>(w.lane);
#pragma unroll
        for (int j = 0; j < 32; j += 4) {
          const float2 x = unpack(acc[16 * c + j / 2]), y = unpack(acc[16 * c + j / 2 + 1]);
          *reinterpret_cast<float4*>(iwp_tc::staged(w.staging, w.lane, j / 4)) = make_float4(x.x, x.y, y.x, y.y);
        }
        while (up.next < c0 + 32) {
          a.z_at[static_cast<int64_t>(row) * a.en.k + up.pos] = *staged_at(w, up.next - c0);
          up.advance(a.en, row);
        }
        __syncwarp();
      }
      if (c0 + 32 > a.V) {
#pragma unroll
        for (int j = 0; j < 32; j += 2) {
          const float2 x = unpack(acc[16 * c + j / 2]);
          acc[16 * c + j / 2] = pack(c0 + j < a.V ? x.x : -CUDART_INF_F, c0 + j + 1 < a.V ? x.y : -CUDART_INF_F);
        }
      }
#pragma unroll
      for (int j = 0; j < 16; j++) {
        const float2 x = unpack(acc[16 * c + j]);
        top = fmaxf(top, fmaxf(x.x, x.y));
      }
    }
    // The maximum is subtracted before the scaling: its own term is then 1 exactly, and a row whose target has all the
    // mass loses nothing, however large its logits are.  Nothing but -inf: sums of 0, not of NaN.
    const float ref = top == -CUDART_INF_F ? 0.f : -top;
    const bool keep = CODES != NO_CODES && w.col0 >= a.v0 && w.col0 < a.v0 + a.width;
    const f2 scale = pack(a.c, a.c), less = pack(ref, ref), up_by = pack(15.f, 15.f);
    const f2 down = pack(-a.c, -a.c), from = pack(8.f + HALF_STEP, 8.f + HALF_STEP);
    f2 sum = pack(0.f, 0.f);
    uint32_t packed[2][16];
#pragma unroll
    for (int c = 0; c < CHUNKS; c++) {
      if (32 * c >= w.width) break;
#pragma unroll
      for (int j = 0; j < 16; j++) {
        const f2 z = add2(acc[16 * c + j], less);
        const float2 x = unpack(fma2(z, scale, up_by));
        const float2 e = make_float2(ex2(x.x), ex2(x.y));
        sum = add2(sum, pack(e.x, e.y));
        if constexpr (CODES == HALF_CODES) packed[c % 2][j] = iwp_tc::pack2(e.x, e.y, IWP_F16);
        if constexpr (CODES == LOG_CODES) {
          const float2 y = unpack(fma2(z, down, from));
          packed[c % 2][j] = log_codes(y.x, y.y);
        }
      }
      if (keep && w.row0 < a.T) {
        if (w.width == 32) {
          iwp_tc::staging_free<0>(w.lane);
          iwp_tc::store_packed(packed[0], w.staging, a.codes, a.ld, w.row0, static_cast<int>(a.T), w.col0 - a.v0, w.lane);
        } else if (c % 2 == 1) {
          copy_out(&a.map, w, packed[0], packed[1], w.col0 + 32 * (c - 1) - a.v0);
        }
      }
    }
    const float2 s = unpack(sum);
    if (live) a.part[static_cast<int64_t>(row) * a.parts + w.col0 / w.width] = make_float2(top, (s.x + s.y) * SUM_SCALE);
  }
};

// ---- epilogue of the probability pass -----------------------------------------------------------------

// Its K is added up in the segments of the logits pass: lse is the sum over the same logits, to the last bit.
struct Probs {
  static constexpr bool SUMS = true;
  static constexpr int AREAS = 2;
  struct Args {
    Targets en;
    const float* lse;
    uint16_t* out;   // [T][ld] of `type`: this piece's columns, and room for what tiles hold beyond them
    int64_t T, ld;
    int v0, width;   // first column of the piece in the vocabulary, columns of the piece
    float c;         // log2(e) / tau
    float up;        // power of two that keeps small probabilities above the smallest fp16 (1 for bf16)
    int type;
    CUtensorMap map; // of `out`, in boxes of 32 rows and 64 columns
  };
  struct Begun {
    Upcoming up;
    float scale, lse2;
  };
  static __device__ __forceinline__ Begun begin(const Args& a, const Where& w) {
    const int row = w.row0 + w.lane;
    Begun b;
    b.up.none(a.en);
    b.scale = b.lse2 = 0.f;
    if (row < a.T) {
      b.scale = a.en.row_scale(row) * a.up;
      b.lse2 = a.lse[row] * LOG2E;
      if (b.scale != 0.f) b.up.from(a.en, row, a.v0 + w.col0);
    }
    return b;
  }
  static __device__ __forceinline__ void tile(const Args& a, Where& w, Begun& begun, f2 (&acc)[iwp_tc::TILE_N / 4]) {
    const int row = w.row0 + w.lane;
    Upcoming& up = begun.up;
    const float scale = begun.scale;
    const f2 c2 = pack(a.c, a.c), less = pack(-begun.lse2, -begun.lse2), scale2 = pack(scale, scale);
    uint32_t packed[2][16];
#pragma unroll
    for (int c = 0; c < iwp_tc::TILE_N / 64; c++) {
      const int c0 = w.col0 + 32 * c;
      if (32 * c >= w.width) break;
      // a row that gives nothing writes zeros whatever its logits are
#pragma unroll
      for (int j = 0; j < 16; j++) {
        const float2 x = unpack(fma2(acc[16 * c + j], c2, less));
        acc[16 * c + j] = scale == 0.f ? pack(0.f, 0.f) : pack(ex2(x.x), ex2(x.y));
      }
      const int end = a.v0 + c0 + 32;
      if (__any_sync(0xFFFFFFFFu, up.next < end)) {  // some row has a target here
        iwp_tc::staging_free<0>(w.lane);
#pragma unroll
        for (int j = 0; j < 32; j += 4) {
          const float2 x = unpack(acc[16 * c + j / 2]), y = unpack(acc[16 * c + j / 2 + 1]);
          *reinterpret_cast<float4*>(iwp_tc::staged(w.staging, w.lane, j / 4)) = make_float4(x.x, x.y, y.x, y.y);
        }
        while (up.next < end) {
          *staged_at(w, up.next - (a.v0 + c0)) -= a.en.q_at(row, up.pos);
          up.advance(a.en, row);
        }
#pragma unroll
        for (int j = 0; j < 32; j += 4) {
          const float4 x = *reinterpret_cast<const float4*>(iwp_tc::staged(w.staging, w.lane, j / 4));
          acc[16 * c + j / 2] = pack(x.x, x.y), acc[16 * c + j / 2 + 1] = pack(x.z, x.w);
        }
        __syncwarp();
      }
#pragma unroll
      for (int j = 0; j < 16; j++) {
        const float2 f = unpack(mul2(acc[16 * c + j], scale2));
        packed[c % 2][j] = iwp_tc::pack2(f.x, f.y, a.type);
      }
      if (w.row0 < a.T && c0 - 32 * (c % 2) < a.width) {
        if (w.width == 32) {
          iwp_tc::staging_free<0>(w.lane);
          iwp_tc::store_packed(packed[0], w.staging, a.out, a.ld, w.row0, static_cast<int>(a.T), c0, w.lane);
        } else if (c % 2 == 1) {
          copy_out(&a.map, w, packed[0], packed[1], c0 - 32);
        }
      }
    }
  }
};

// ---- epilogue of the gradient products ------------------------------------------------------------------

// What both gradients are multiplied with: `factor` (scale * tau / up) * dloss / n.
struct Factor {
  const Header* hdr;
  const float* dloss;
  float factor;
  int mean;
  __device__ __forceinline__ float get() const {
    float f = factor;
    if (dloss) f *= *dloss;
    if (mean) f /= static_cast<float>(max(hdr->n_rows, 1));
    return f;
  }
};

struct OutMatrix {
  void* out;
  int64_t ld, split_stride;  // elements
  int rows, cols, type, wide, add, raw;  // raw: partial sums, the factor is applied later
  int by_copy;                           // 16-bit rows that start at multiples of 16 bytes, nothing to add
  int by_gmax;                           // dweight, where the hidden states carry the rows' powers of two
  const float* row_power;                // dhidden: [rows], or NULL
  CUtensorMap map;                       // of `out` then, in boxes of 32 rows and 64 columns
};

struct OutArgs {
  Factor f;
  OutMatrix m[2];
};

// LONG: for K of several segments, whose sums are in registers and leave fewer of them to the stores: 3001 x 8060 x 1031 takes
// 200 us with them and 193 without, so products of one segment do without.
template <bool LONG>
struct Out {
  static constexpr bool SUMS = LONG;
  static constexpr int AREAS = 2;
  using Args = OutArgs;
  static __device__ __forceinline__ float begin(const Args& args, const Where& w) {
    const OutMatrix& a = args.m[w.p];
    if (a.raw) return 1.f;
    const float f = args.f.get();
    if (a.by_gmax) return f * args.f.hdr->gmax;
    return a.row_power && w.row0 + w.lane < a.rows ? f * a.row_power[w.row0 + w.lane] : f;
  }
  using Sums = std::conditional_t<LONG, f2 (&)[iwp_tc::TILE_N / 4], uint32_t>;
  // 32 of the warp's columns, from c on, times f; in registers c is a constant
  static __device__ __forceinline__ void take(Sums sums, int c, float f, float (&v)[32]) {
    if constexpr (LONG) {
#pragma unroll
      for (int j = 0; j < 16; j++) {
        const float2 x = unpack(mul2(sums[c / 2 + j], pack(f, f)));
        v[2 * j] = x.x, v[2 * j + 1] = x.y;
      }
    } else {
      iwp_tc::tmem_load32(sums + c, v);
#pragma unroll
      for (int j = 0; j < 32; j++) v[j] *= f;
    }
  }
  static __device__ __forceinline__ void copy64(const OutMatrix& a, Where& w, float f, Sums sums, int c) {
    uint32_t packed[2][16];
#pragma unroll
    for (int half = 0; half < 2; half++) {
      float v[32];
      take(sums, c + 32 * half, f, v);
#pragma unroll
      for (int j = 0; j < 16; j++) packed[half][j] = iwp_tc::pack2(v[2 * j], v[2 * j + 1], a.type);
    }
    // (the accumulator is read whole all the same: a warp's loads are collective)
    if (w.row0 < a.rows) copy_out(&a.map, w, packed[0], packed[1], w.col0 + c);
  }
  static __device__ __forceinline__ void tile(const Args& args, Where& w, float f, Sums sums) {
    const OutMatrix& a = args.m[w.p];
    const int end = min(w.width, a.cols - w.col0);
    if (a.by_copy && w.width >= 64) {
      if constexpr (LONG) {
#pragma unroll
        for (int c = 0; c < iwp_tc::TILE_N / 2; c += 64)
          if (c < end) copy64(a, w, f, sums, c);
      } else {
#pragma unroll 1
        for (int c = 0; c < end; c += 64) copy64(a, w, f, sums, c);
      }
      return;
    }
    iwp_tc::staging_free<0>(w.lane);
    char* const out = static_cast<char*>(a.out) + w.split * a.split_stride * (a.type == IWP_F32 ? 4 : 2);
    const bool half = a.type != IWP_F32 && !a.add;  // staged in 16 bits
    // 64 columns at a time, after which the sums in registers move up: one copy of the many ways to store, and room for it
#pragma unroll 1
    for (int c = 0; c < end; c += 64) {
#pragma unroll
      for (int i = 0; i < 64; i += 32) {
        if (c + i < end) {
          float v[32];
          take(sums, LONG ? i : c + i, f, v);
          if (half)
            iwp_tc::stage_chunk(v, w.staging, w.lane, i / 8, a.type);
          else
            iwp_tc::stage_chunk(v, w.staging + i / 32 * iwp_tc::STAGING_BYTES, w.lane);
        }
      }
      if constexpr (LONG) {
#pragma unroll
        for (int j = 0; j < 32; j++) sums[j] = sums[j + 32];
      }
      __syncwarp();
      if (half) {
        if (w.row0 < a.rows)
          iwp_tc::write_rows16(w.staging, reinterpret_cast<uint16_t*>(out) + w.row0 * a.ld + w.col0 + c, a.ld, a.wide, w.row0, a.rows, min(64, end - c),
                               w.lane);
        __syncwarp();
        continue;
      }
#pragma unroll 1
      for (int i = 0; i < min(64, end - c); i += 32)
        iwp_tc::write_chunk<LONG ? 4 : 8>(w.staging + i / 32 * iwp_tc::STAGING_BYTES, out, a.ld, a.type, a.wide, a.add, w.row0, a.rows, w.col0 + c + i, a.cols, w.lane);
      __syncwarp();
    }
  }
};

// dhidden = factor (* the row's power of two) * sum over the splits (in order), rounded once.  The parts' rows hold whole groups of four columns; a
// thread takes a group.  Bound by latency for the sizes that are split at all (1021 x 1032 in two parts: 7 us).
__global__ void __launch_bounds__(256) k_join(Factor f, const float* row_power, const float* part, int splits, int64_t rows, int cols, void* out,
                                              int64_t ld, int type, int add, int wide) {
  iwp_tc::launch_next();
  iwp_tc::wait_previous();
  const float all = f.get();
  const int groups = (cols + 3) / 4;
  const int64_t n = rows * groups * 4;
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const float k = row_power ? all * row_power[r] : all;
    for (int g = threadIdx.x; g < groups; g += blockDim.x) {
      const int64_t i = (r * groups + g) * 4, at = r * ld + 4 * g;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int s = 0; s < splits; s++) {
        const float4 y = __ldcs(reinterpret_cast<const float4*>(part + s * n + i));
        x.x += y.x, x.y += y.y, x.z += y.z, x.w += y.w;
      }
      float v[4] = {x.x * k, x.y * k, x.z * k, x.w * k};
      const int have = min(4, cols - 4 * g);
      if (add)
        for (int j = 0; j < have; j++) v[j] += iwp_tc::load_as_float(out, at + j, type);
      if (!wide || have < 4) {
        for (int j = 0; j < have; j++) iwp_tc::store_as(out, at + j, v[j], type);
      } else if (type == IWP_F32) {
        *reinterpret_cast<float4*>(static_cast<float*>(out) + at) = make_float4(v[0], v[1], v[2], v[3]);
      } else {
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + at) =
            make_uint2(iwp_tc::pack2(v[0], v[1], type), iwp_tc::pack2(v[2], v[3], type));
      }
    }
  }
}

// ---- targets -----------------------------------------------------------------------------------------------

__device__ __forceinline__ int64_t load_id(const void* ids, int64_t i, int bytes) {
  return bytes == 8 ? static_cast<const int64_t*>(ids)[i] : static_cast<const int32_t*>(ids)[i];
}

__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
  return x;
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
  return x;
}

// One warp per row: softmax over the row's teacher logits; entries ordered by column (by counting the smaller ones: top_k^2
// comparisons in shared memory, less than a sort costs up to about a hundred), equal ids joined into one.  4096 x 64: 12 us.
__global__ void k_soft_targets(int* column, float* q_out, float* const_term, const void* ids, int64_t ids_ld, int ids_bytes,
                               const void* logits, int64_t logits_ld, int type, int K, float inv_tau, int64_t T, int64_t V) {
  extern __shared__ int sh[];
  iwp_tc::wait_previous();
  iwp_tc::launch_next();  // after the wait: the logits pass may load its operands beside this kernel
  const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t t = blockIdx.x * int64_t(warps) + warp;
  if (t >= T) return;
  int* col = sh + warp * 2 * K;
  float* q = reinterpret_cast<float*>(col + K);
  float top = -CUDART_INF_F;
  bool bad = false, nan = false;
  for (int k = lane; k < K; k += 32) {
    const int64_t id = load_id(ids, t * ids_ld + k, ids_bytes);
    const float x = iwp_tc::load_as_float(logits, t * logits_ld + k, type);
    bad |= id >= V;
    const bool used = id >= 0 && id < V && x != -CUDART_INF_F;  // NaN takes part
    col[k] = used ? static_cast<int>(id) : NO_COLUMN;
    q[k] = x;
    if (used) {
      nan |= x != x;
      top = fmaxf(top, x);
    }
  }
  bad = __any_sync(0xFFFFFFFFu, bad);
  nan = __any_sync(0xFFFFFFFFu, nan);
  top = warp_max(top);
  __syncwarp();
  float sum = 0.f;
  for (int k = lane; k < K; k += 32)
    if (col[k] != NO_COLUMN) sum += expf((q[k] - top) * inv_tau);  // subtracted first: a type's lowest value, over tau, leaves it
  sum = warp_sum(sum);
  const bool has = top != -CUDART_INF_F || nan;
  const float log_sum = logf(sum);
  float term = 0.f;
  for (int k = lane; k < K; k += 32) {
    float p = 0.f;
    if (col[k] != NO_COLUMN) {
      const float lq = (q[k] - top) * inv_tau - log_sum;
      p = expf(lq);
      if (p != 0.f) term += p * lq;
    }
    q[k] = p;
  }
  term = warp_sum(term);
  __syncwarp();
  for (int k = lane; k < K; k += 32) {
    const int c = col[k];
    int rank = 0, before = 0;
    float p = 0.f;
    for (int j = 0; j < K; j++) {
      const int o = col[j];
      rank += o < c || (o == c && j < k);
      before += o == c && j < k;
      if (o == c) p += q[j];
    }
    // of equal ids the first carries the sum, the others stay in place with nothing: the order is kept
    const bool drop = c == NO_COLUMN;
    column[t * K + rank] = bad || drop ? NO_COLUMN : c;
    q_out[t * K + rank] = drop || before ? 0.f : p;
  }
  if (lane == 0) const_term[t] = bad ? CUDART_NAN_F : has ? term : 0.f;
}

// ---- per-row upstream gradients of fp16 operands ------------------------------------------------------------------
//
// bf16 factors take the rows' upstream gradients directly: they have fp32's range.  In fp16 a row far below the others'
// would lose its small probabilities, and with them its own gradient, which does not depend on the others'.  There an
// upstream gradient is split as r 2^e, 1 <= |r| < 2: the factors take r; dhidden's epilogue takes the row's 2^e; for
// dweight, a sum over the rows, a copy of the hidden states takes 2^e relative to the largest of them (its small rows may
// be rounded to fp16's smallest steps, which are 2^-24 beside the large rows' values; rows that give nothing are zero).
__global__ void __launch_bounds__(1024) k_row_scales(Header* hdr, Targets en, float* scale, float* power, const float* dloss_rows, int64_t T) {
  __shared__ float sh[32];
  iwp_tc::launch_next();
  iwp_tc::wait_previous();
  float top = 0.f;
  for (int64_t t = threadIdx.x; t < T; t += blockDim.x) {
    float r = en.state(t) == 1 ? dloss_rows[t] : 0.f, p = 1.f;
    if (r != 0.f && isfinite(r)) {
      int e;
      r = 2.f * frexpf(r, &e);
      p = ldexpf(1.f, e - 1);
      top = fmaxf(top, p);
    }
    scale[t] = r;
    power[t] = p;
  }
  top = warp_max(top);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = top;
  __syncthreads();
  top = warp_max(sh[threadIdx.x & 31]);
  if (threadIdx.x == 0) hdr->gmax = top > 0.f ? top : 1.f;
}

// The copy of the hidden states for dweight; rows of both start at multiples of 16 bytes.  A warp takes a row.
__global__ void __launch_bounds__(256) k_scaled_rows(const Header* hdr, const float* scale, const float* power, const __half* from, int64_t ld_from,
                                                     __half* to, int64_t ld_to, int64_t rows, int cols) {
  iwp_tc::launch_next();
  iwp_tc::wait_previous();
  const int lane = threadIdx.x & 31;
  const float all = hdr->gmax;
  for (int64_t r = blockIdx.x * 8ll + (threadIdx.x >> 5); r < rows; r += gridDim.x * 8ll) {
    const bool gives = scale[r] != 0.f;
    const float k = power[r] / all;
    for (int g = 8 * lane; g < cols; g += 8 * 32) {
      union {
        __half e[8];
        uint4 all;
      } x;
      if (g + 8 <= cols) {
        x.all = *reinterpret_cast<const uint4*>(from + r * ld_from + g);
      } else {
#pragma unroll
        for (int j = 0; j < 8; j++) x.e[j] = g + j < cols ? from[r * ld_from + g + j] : __float2half_rn(0.f);
      }
#pragma unroll
      for (int j = 0; j < 8; j++) x.e[j] = __float2half_rn(gives ? __half2float(x.e[j]) * k : 0.f);
      *reinterpret_cast<uint4*>(to + r * ld_to + g) = x.all;
    }
  }
}

// dweight sums over all rows, and zero times what is not finite is not zero: where a row that gives nothing (padding, say, that
// attended to nothing) holds NaN or infinities, which its lse tells, the product reads a copy of the hidden states in
// which such rows are zero.  Rows of both start at multiples of 16 bytes.  A warp takes a row.
struct Clean {
  const uint16_t* from;
  uint16_t* to;  // NULL: not needed
  int64_t ld_from, ld_to, T;
  int D;
};
__device__ __forceinline__ void clean_rows(const Clean& a, const Targets& en, int64_t warp, int64_t warps) {
  const int lane = threadIdx.x & 31;
  for (int64_t r = warp; r < a.T; r += warps) {
    const bool gives = en.row_scale(r) != 0.f;
    for (int g = 8 * lane; g < a.D; g += 8 * 32) {
      union {
        uint16_t e[8];
        uint4 all;
      } x;
      x.all = make_uint4(0u, 0u, 0u, 0u);
      if (gives && g + 8 <= a.D) {
        x.all = *reinterpret_cast<const uint4*>(a.from + r * a.ld_from + g);
      } else if (gives) {
#pragma unroll
        for (int j = 0; j < 8; j++)
          if (g + j < a.D) x.e[j] = a.from[r * a.ld_from + g + j];
      }
      *reinterpret_cast<uint4*>(a.to + r * a.ld_to + g) = x.all;
    }
  }
}

// Number of rows with targets, and whether one is outside the vocabulary, for backward passes on their own (k_rows sees to
// both otherwise); the same for clean_rows, by its one block.
__global__ void __launch_bounds__(1024) k_count_rows(Header* hdr, Targets en, const float* lse, Clean copy, int64_t T) {
  __shared__ int sh[32];
  iwp_tc::launch_next();
  iwp_tc::wait_previous();
  int n = 0;
  bool bad = false, dirty = false;
  for (int64_t t = threadIdx.x; t < T; t += blockDim.x) {
    const int state = en.state(t);
    n += state != 0;
    bad |= state < 0;
    dirty |= !isfinite(lse[t]) && en.row_scale(t) == 0.f;
  }
  if (bad) atomicExch(&hdr->status, IWP_ERR_INVALID);
  n = __reduce_add_sync(0xFFFFFFFFu, n);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = n;
  __syncthreads();
  n = __reduce_add_sync(0xFFFFFFFFu, sh[threadIdx.x & 31]);
  dirty = __syncthreads_or(dirty && copy.to);
  if (threadIdx.x == 0) hdr->n_rows = n, hdr->clean = dirty;
  if (dirty) clean_rows(copy, en, threadIdx.x >> 5, blockDim.x >> 5);
}

// ---- finish of the forward pass --------------------------------------------------------------------------

struct Rows {
  Header* hdr;
  Targets en;
  const float2* part;  // [T][parts]
  const float* z_at;
  float* rows;  // the caller's, or scratch
  float* lse;
  float* loss;
  int64_t T;
  int parts, lanes, mean;
  float tau, c;  // log2(e) / tau
};

constexpr int ROW_THREADS = 256;

__device__ __forceinline__ float2 join(float2 a, float2 b, float c) {  // (maximum, sum of 2^((z - maximum) c))
  const float m = fmaxf(a.x, b.x), ref = m == -CUDART_INF_F ? 0.f : m;
  return make_float2(m, a.y * ex2((a.x - ref) * c) + b.y * ex2((b.x - ref) * c));
}

// lse and loss of a row by a warp (lanes = 32), or by the block where there are few rows (lanes = 256); the last block to
// finish adds the rows' losses in a fixed order.  Bound by the latency of four dependent reads and the ticket: 7 us for up to
// a few hundred rows, 13 for 4096 rows of 256 parts.
__global__ void __launch_bounds__(ROW_THREADS) k_rows(const Rows a) {
  constexpr int WARPS = ROW_THREADS / 32;
  __shared__ float2 sh[WARPS];
  __shared__ float sh_sum[WARPS];
  __shared__ int sh_n[WARPS];
  __shared__ bool last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  iwp_tc::wait_previous();
  iwp_tc::launch_next();  // after the wait: whoever runs beside this kernel may read what the logits pass left
  const int64_t row = a.lanes == 32 ? blockIdx.x * int64_t(WARPS) + warp : blockIdx.x;
  const int me = a.lanes == 32 ? lane : tid;
  if (row < a.T) {
    // the row's target of this lane, fetched beside the parts
    int column = NO_COLUMN;
    float q = 0.f, z = 0.f;
    if (me < a.en.k) {
      column = a.en.column_at(row, me);
      q = a.en.q_at(row, me);
      if (column != NO_COLUMN) z = a.z_at[row * a.en.k + me];
    }
    const int state = a.en.state(row);
    const float2* const part = a.part + row * a.parts;
    float2 x = make_float2(-CUDART_INF_F, 0.f);
#pragma unroll 4
    for (int p = me; p < a.parts; p += a.lanes) x = join(x, part[p], a.c);
#pragma unroll
    for (int o = 16; o; o >>= 1) x = join(x, make_float2(__shfl_xor_sync(0xFFFFFFFFu, x.x, o), __shfl_xor_sync(0xFFFFFFFFu, x.y, o)), a.c);
    if (a.lanes != 32) {
      if (lane == 0) sh[warp] = x;
      __syncthreads();
      x = sh[0];
#pragma unroll
      for (int w = 1; w < WARPS; w++) x = join(x, sh[w], a.c);
    }
    // q (lse - z / tau) entry by entry and without lse, whose last bits a large logit takes: the sum is 1 or more and
    // the maximum no less than z, so the loss of a confident row is small and never negative
    const float log_sum = logf(x.y);
    float below = column != NO_COLUMN && q != 0.f ? q * ((x.x - z) / a.tau + log_sum) : 0.f;
    for (int k = me + a.lanes; k < a.en.k; k += a.lanes) {
      if (a.en.column_at(row, k) == NO_COLUMN) break;
      const float qk = a.en.q_at(row, k);
      if (qk != 0.f) below += qk * ((x.x - a.z_at[row * a.en.k + k]) / a.tau + log_sum);
    }
    below = warp_sum(below);
    if (a.lanes != 32) {
      if (lane == 0) sh_sum[warp] = below;
      __syncthreads();
      below = 0.f;
      for (int w = 0; w < WARPS; w++) below += sh_sum[w];
      __syncthreads();
    }
    if (me == 0) {
      const float c = a.en.hard ? 0.f : a.en.const_term[row];
      const float lse = x.x / a.tau + log_sum;
      a.lse[row] = lse;
      if (!isfinite(lse) && a.en.row_scale(row) == 0.f) atomicExch(&a.hdr->dirty, 1);
      a.rows[row] = state == 0 ? 0.f : state < 0 ? CUDART_NAN_F : a.tau * a.tau * (c + below);
      if (state < 0) atomicExch(&a.hdr->status, IWP_ERR_INVALID);
      __threadfence();
    }
  }
  __syncthreads();
  if (tid == 0) last = gridDim.x == 1 || atomicInc(&a.hdr->ticket, gridDim.x - 1) == gridDim.x - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  float sum = 0.f;
  int n = 0;
#pragma unroll 4
  for (int64_t t = tid; t < a.T; t += ROW_THREADS) {
    sum += __ldcg(a.rows + t);
    n += a.en.state(t) != 0;
  }
  sum = warp_sum(sum);
  n = __reduce_add_sync(0xFFFFFFFFu, n);
  if (lane == 0) sh_sum[warp] = sum, sh_n[warp] = n;
  __syncthreads();
  if (tid == 0) {
    sum = 0.f, n = 0;
    for (int w = 0; w < WARPS; w++) sum += sh_sum[w], n += sh_n[w];
    a.hdr->n_rows = n;
    a.hdr->clean = atomicExch(&a.hdr->dirty, 0);
    if (a.loss) *a.loss = n == 0 ? 0.f : a.mean ? sum / static_cast<float>(n) : sum;
  }
}

// ---- codes of the kept piece -> factors ------------------------------------------------------------------------

struct Factors {
  Targets en;
  const float2* part;  // [T][parts]
  const float* z_at;   // [T][k] logits at the targets
  const float* lse;
  uint16_t* codes;  // [T][ld], in place
  int64_t ld;
  int parts, part_shift, v0, width, chunks, log_codes;
  float c, up;  // log2(e) / tau
  const Header* hdr;
  int64_t blocks;  // of the factors; any others clean_rows, if there is need
  Clean copy;
};

constexpr int FACTOR_THREADS = 256, FACTOR_DEEP = 4, FACTOR_COLUMNS = 8 * FACTOR_THREADS * FACTOR_DEEP;

// A block takes FACTOR_COLUMNS columns of one row: bound by memory, 2 bytes in and 2 out per element (4096 x 32768: 78 us =
// 6.9 TB/s with the end of the codes still in the L2; with 64 targets per row to look through, 90 us).
__global__ void __launch_bounds__(FACTOR_THREADS) k_factors(const Factors a) {
  constexpr int MINE = (MAX_TOP + FACTOR_THREADS - 1) / FACTOR_THREADS, WARPS = FACTOR_THREADS / 32;
  const int tid = threadIdx.x;
  if (blockIdx.x >= a.blocks) {
    iwp_tc::launch_next();
    iwp_tc::wait_previous();
    if (a.hdr->clean) clean_rows(a.copy, a.en, (blockIdx.x - a.blocks) * WARPS + tid / 32, (gridDim.x - a.blocks) * WARPS);
    return;
  }
  const int64_t row = blockIdx.x / a.chunks;
  uint16_t* const codes = a.codes + row * a.ld;
  const float2* const part = a.part + row * a.parts;
  const int c0 = static_cast<int>(blockIdx.x - row * a.chunks) * FACTOR_COLUMNS, c1 = min(c0 + FACTOR_COLUMNS, a.width);
  iwp_tc::launch_next();
  // what the logits pass and the targets' kernel left is complete: k_rows started after them, and this kernel after that
  uint4 u[FACTOR_DEEP];
  float m[FACTOR_DEEP];
#pragma unroll
  for (int i = 0; i < FACTOR_DEEP; i++) {
    const int o = c0 + 8 * tid + i * 8 * FACTOR_THREADS;
    if (o < c1) {
      u[i] = *reinterpret_cast<const uint4*>(codes + o);
      m[i] = part[(a.v0 + o) >> a.part_shift].x;
    }
  }
  const float scale = a.en.row_scale(row) * a.up;
  int at[MINE];
  float z[MINE];
  bool any = false;
#pragma unroll
  for (int i = 0; i < MINE; i++) {
    const int k = tid + i * FACTOR_THREADS;
    at[i] = -1;
    if (k < a.en.k) {
      const int col = a.en.column_at(row, k);
      if (col >= a.v0 + c0 && col < a.v0 + c1 && a.en.q_at(row, k) != 0.f) {
        at[i] = col - a.v0;
        z[i] = a.z_at[row * a.en.k + k];
        any = true;
      }
    }
  }
  iwp_tc::wait_previous();
  const float lse2 = a.lse[row] * LOG2E;
  any = __syncthreads_or(any);
#pragma unroll
  for (int i = 0; i < FACTOR_DEEP; i++) {
    const int o = c0 + 8 * tid + i * 8 * FACTOR_THREADS;
    if (o >= c1) break;
    uint32_t* const e = reinterpret_cast<uint32_t*>(&u[i]);
    const float top = fmaf(m[i], a.c, -lse2);  // the part's maximum less lse, in log2
    if (scale == 0.f) {  // a row that gives nothing, whatever its logits are
      u[i] = make_uint4(0u, 0u, 0u, 0u);
    } else if (a.log_codes) {
#pragma unroll
      for (int j = 0; j < 4; j++)
        e[j] = iwp_tc::pack2(ex2(top + 8.f - log_value(e[j] & 0xFFFFu)) * scale, ex2(top + 8.f - log_value(e[j] >> 16)) * scale, IWP_F16);
    } else {
      const float f = ex2(top - 15.f) * scale;
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const float2 x = iwp_tc::unpack2(e[j], IWP_F16);
        e[j] = iwp_tc::pack2(x.x * f, x.y * f, IWP_BF16);
      }
    }
    *reinterpret_cast<uint4*>(codes + o) = u[i];
  }
  if (!any || scale == 0.f) return;
  __syncthreads();  // the factors of columns without a target are there
  // p - q cancels where a student is close to its teacher: p of a target comes from its fp32 logit, not from its code
#pragma unroll
  for (int i = 0; i < MINE; i++)
    if (at[i] >= 0) {
      const float p = ex2(fmaf(z[i], a.c, -lse2));
      iwp_tc::store_as(codes, at[i], (p - a.en.q_at(row, tid + i * FACTOR_THREADS)) * scale, a.log_codes ? IWP_F16 : IWP_BF16);
    }
}

// ---- forward pass of a few tokens -------------------------------------------------------------------------------

struct Few {
  Targets en;
  const void* hidden;
  const void* weight;
  float2* part;  // [T][blocks]
  float* z_at;
  int64_t hidden_ld, weight_ld;
  int T, V, D, type, blocks;  // the first `blocks` blocks share the vocabulary, the others take the targets' logits
  float c;
};

constexpr int FEW_TOKENS = 2, FEW_THREADS = 512, FEW_ROWS = 4;

// Four rows of the weights per warp at a time, streamed once: dot products with one or two tokens are bound by the weights'
// bytes, and plain loads keep more of them in flight than the tensor cores' 128-row tiles would (131072 x 4096, one token:
// 165 us = 6.5 TB/s, against 253 by tiles; two tokens 183 and 214; from three on, tiles are as fast).  A group of 8
// elements is widened once per row and once per token.  Operand rows start at multiples of 16 bytes and hold whole ones
// (copies made by k_align_rows end in zeros).
template <int TOKENS>
__global__ void __launch_bounds__(FEW_THREADS, 2) k_few_tokens(const Few a) {
  constexpr int WARPS = FEW_THREADS / 32;
  extern __shared__ uint4 sh_hidden[];  // [TOKENS][D / 8, rounded up]
  __shared__ float2 sh[WARPS][TOKENS];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int groups = (a.D + 7) / 8;
  iwp_tc::launch_next();
  const uint16_t* const hidden = static_cast<const uint16_t*>(a.hidden);
  const uint16_t* const weight = static_cast<const uint16_t*>(a.weight);
  // the beginning (2 KB each) of this warp's first rows is on its way to the L2 while the kernel before this one ends
  for (int i = lane; i < FEW_ROWS * 16; i += 32) {
    const int v = (blockIdx.x * WARPS + warp) * FEW_ROWS + i / 16;
    if (static_cast<int>(blockIdx.x) < a.blocks && v < a.V && 8 * (i % 16) < groups)
      asm volatile("prefetch.global.L2 [%0];" ::"l"(weight + v * a.weight_ld + 64 * (i % 16)));
  }
  iwp_tc::wait_previous();
  for (int i = tid; i < TOKENS * groups; i += FEW_THREADS) {
    const int t = i / groups, g = i - t * groups;
    sh_hidden[i] = *reinterpret_cast<const uint4*>(hidden + t * a.hidden_ld + 8 * g);
  }
  __syncthreads();
  auto load8 = [&](const uint16_t* row, int g) { return __ldcs(reinterpret_cast<const uint4*>(row + 8 * g)); };
  auto widen = [&](const uint4& x, f2 (&y)[4]) {
    const uint32_t* const e = reinterpret_cast<const uint32_t*>(&x);
#pragma unroll
    for (int j = 0; j < 4; j++) {
      const float2 v = iwp_tc::unpack2(e[j], a.type);
      y[j] = pack(v.x, v.y);
    }
  };
  if (static_cast<int>(blockIdx.x) >= a.blocks) {  // logits at the targets, a warp each
    const int i = (blockIdx.x - a.blocks) * WARPS + warp;
    if (i >= a.T * a.en.k) return;
    const int t = i / a.en.k, col = a.en.column_at(t, i - t * a.en.k);
    if (col == NO_COLUMN) return;
    f2 acc = pack(0.f, 0.f);
    for (int g = lane; g < groups; g += 32) {
      f2 x[4], y[4];
      widen(load8(weight + col * a.weight_ld, g), x);
      widen(sh_hidden[t * groups + g], y);
#pragma unroll
      for (int j = 0; j < 4; j++) acc = fma2(x[j], y[j], acc);
    }
    const float z = warp_sum(unpack(acc).x + unpack(acc).y);
    if (lane == 0) a.z_at[i] = z;
    return;
  }
  float m[TOKENS], s[TOKENS];
#pragma unroll
  for (int t = 0; t < TOKENS; t++) m[t] = -CUDART_INF_F, s[t] = 0.f;
  for (int v = (blockIdx.x * WARPS + warp) * FEW_ROWS; v < a.V; v += a.blocks * WARPS * FEW_ROWS) {
    f2 acc[FEW_ROWS][TOKENS];
#pragma unroll
    for (int r = 0; r < FEW_ROWS; r++)
#pragma unroll
      for (int t = 0; t < TOKENS; t++) acc[r][t] = pack(0.f, 0.f);
    const uint16_t* const row = weight + v * a.weight_ld;
    const int have = min(FEW_ROWS, a.V - v);
#pragma unroll 2
    for (int g = lane; g < groups; g += 32) {
      uint4 w[FEW_ROWS];
#pragma unroll
      for (int r = 0; r < FEW_ROWS; r++) w[r] = load8(row + min(r, have - 1) * a.weight_ld, g);
      f2 y[TOKENS][4];
#pragma unroll
      for (int t = 0; t < TOKENS; t++) widen(sh_hidden[t * groups + g], y[t]);
#pragma unroll
      for (int r = 0; r < FEW_ROWS; r++) {
        f2 x[4];
        widen(w[r], x);
#pragma unroll
        for (int t = 0; t < TOKENS; t++)
#pragma unroll
          for (int j = 0; j < 4; j++) acc[r][t] = fma2(x[j], y[t][j], acc[r][t]);
      }
    }
#pragma unroll
    for (int t = 0; t < TOKENS; t++) {
      float z[FEW_ROWS], top = m[t];
#pragma unroll
      for (int r = 0; r < FEW_ROWS; r++) {
        const float2 both = unpack(acc[r][t]);
        z[r] = warp_sum(both.x + both.y);
        if (r >= have) z[r] = -CUDART_INF_F;
        top = fmaxf(top, z[r]);
      }
      const float ref = top == -CUDART_INF_F ? 0.f : top;
      s[t] *= ex2((m[t] - ref) * a.c);
#pragma unroll
      for (int r = 0; r < FEW_ROWS; r++) s[t] += ex2((z[r] - ref) * a.c);
      m[t] = top;
    }
  }
  if (lane == 0)
#pragma unroll
    for (int t = 0; t < TOKENS; t++) sh[warp][t] = make_float2(m[t], s[t]);
  __syncthreads();
  if (tid < TOKENS) {
    float2 x = sh[0][tid];
    for (int w = 1; w < WARPS; w++) x = join(x, sh[w][tid], a.c);
    a.part[tid * a.blocks + blockIdx.x] = x;
  }
}

// Rows of `cols` 16-bit elements to rows of `ld_to` (a multiple of 8; zeros at the end), for operands TMA cannot address.
// A warp takes a row, a lane 16 bytes of the result at a time, read in the widest units that all rows start on.  Bound by
// memory.
template <class Unit>
__global__ void __launch_bounds__(256) k_align_rows(const uint16_t* from, int64_t ld_from, uint16_t* to, int64_t ld_to, int64_t rows, int cols) {
  constexpr int PER = sizeof(Unit) / 2, UNITS = 8 / PER;
  iwp_tc::launch_next();
  iwp_tc::wait_previous();
  const int lane = threadIdx.x & 31, groups = static_cast<int>(ld_to / 8);
  for (int64_t r = blockIdx.x * 8ll + (threadIdx.x >> 5); r < rows; r += gridDim.x * 8ll) {
    const uint16_t* const row = from + r * ld_from;
#pragma unroll 2
    for (int g = lane; g < groups; g += 32) {
      union {
        Unit u[UNITS];
        uint16_t e[8];
        uint4 all;
      } x;
      x.all = make_uint4(0u, 0u, 0u, 0u);
      if (8 * g + 8 <= cols) {
#pragma unroll
        for (int j = 0; j < UNITS; j++) x.u[j] = *reinterpret_cast<const Unit*>(row + 8 * g + PER * j);
      } else {
#pragma unroll
        for (int j = 0; j < 8; j++)
          if (8 * g + j < cols) x.e[j] = row[8 * g + j];
      }
      *reinterpret_cast<uint4*>(to + r * ld_to + 8 * g) = x.all;
    }
  }
}

}  // namespace iwp_head
