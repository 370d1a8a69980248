// iwp_head.cuh - output head with its loss (cross entropy, or a teacher's top logits): what happens to the tiles of
// the three products of iwp_tensor.cuh, and the small kernels around them.
//
//   logits pass   z tile -> per row and 128 columns: maximum and sum of exp (written), the logits at the targets
//   finish        per row: lse, loss; their sum in a fixed order
//   probability   z tile again (recomputed: 2 D operations per logit cost less than keeping T x V of them) ->
//   pass          row_scale * (exp(z / tau - lse) - q), rounded to the operands' type, for one piece of the vocabulary
//   dweight       P^T hidden for the piece: complete, since the piece holds every token
//   dhidden       P weight for the piece, summed over the pieces in fp32
//
// Cross entropy and distillation differ only in the list of (column, q) that each row subtracts: one entry or top_k
// of them, sorted by column, so that an epilogue warp meets them in the order in which it walks the columns.
#pragma once

#include <math_constants.h>

#include "../../include/iwp_loss.h"
#include "iwp_tensor.cuh"

namespace iwp_head {

using iwp_tc::Tile;

constexpr int MAX_TOP = 1024;
constexpr int NO_COLUMN = 0x7FFFFFFF;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// First bytes of a workspace.
struct Header {
  int status;
  int n_rows;       // rows with targets
  uint32_t ticket;  // blocks of the finish kernel that are done
  float gmax;       // largest |dloss_rows|
};

struct Entries {  // sorted by column within a row; unused ones are NO_COLUMN at the end.  [k][T]: lanes are rows
  int* column;
  float* q;
  float* const_term;  // [T] sum of q log q; NaN for a row with a target outside the vocabulary
  float* row_scale;   // [T] 1 for a row that gives gradients, 0 otherwise; dloss_rows / gmax where those are given
  int k;
};

__device__ __forceinline__ int first_entry(const Entries& en, int64_t T, int row, int col0) {
  int lo = 0, hi = en.k;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (en.column[mid * T + row] < col0)
      lo = mid + 1;
    else
      hi = mid;
  }
  return lo;
}

// ---- epilogue of the logits pass --------------------------------------------------------------------

struct Logits {
  struct Args {
    Entries en;
    int64_t T;
    int V;
    float c;          // log2(e) / tau
    float2* part;     // [2 * n_tiles][T]: maximum (of z * c) and sum of 2^(z c - maximum)
    float* z_at;      // [k][T] logits at the targets
  };
  static __device__ __forceinline__ void tile(const Args& a, const Tile& t, uint32_t tmem, int row_block, int e, int lane,
                                              char* staging) {
    const int row = row_block * iwp_tc::TILE_M + (e % 4) * 32 + lane;
    const bool live = row < a.T;
    const int part = 2 * t.n + e / 4, col0 = part * (iwp_tc::TILE_N / 2);
    int pos = 0, next = NO_COLUMN;
    if (live) {
      pos = first_entry(a.en, a.T, row, col0);
      if (pos < a.en.k) next = a.en.column[pos * a.T + row];
    }
    float m = -CUDART_INF_F, s = 0.f;
#pragma unroll 1
    for (int c0 = col0; c0 < min(col0 + iwp_tc::TILE_N / 2, a.V); c0 += 32) {
      float v[32];
      iwp_tc::tmem_load32(tmem + (c0 - col0), v);
      if (__any_sync(0xFFFFFFFFu, next < c0 + 32)) {  // some row has a target here
        float* mine = reinterpret_cast<float*>(staging + lane * iwp_tc::STAGING_PITCH);
#pragma unroll
        for (int j = 0; j < 32; j += 4) *reinterpret_cast<float4*>(mine + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
        while (next < c0 + 32) {
          a.z_at[pos * a.T + row] = mine[next - c0];
          pos++;
          next = pos < a.en.k ? a.en.column[pos * a.T + row] : NO_COLUMN;
        }
        __syncwarp();
      }
      if (c0 + 32 > a.V) {
#pragma unroll
        for (int j = 0; j < 32; j++)
          if (c0 + j >= a.V) v[j] = -CUDART_INF_F;
      }
      float top = v[0];
#pragma unroll
      for (int j = 1; j < 32; j++) top = fmaxf(top, v[j]);
      const float m_new = fmaxf(m, top * a.c);
      const float ref = m_new == -CUDART_INF_F ? 0.f : m_new;
      float add = 0.f;
#pragma unroll
      for (int j = 0; j < 32; j++) add += exp2f(fmaf(v[j], a.c, -ref));
      s = s * exp2f(m - ref) + add;
      m = m_new;
    }
    if (live) a.part[part * a.T + row] = make_float2(m, s);
  }
};

// ---- epilogue of the probability pass -----------------------------------------------------------------

struct Probs {
  struct Args {
    Entries en;
    const float* lse;
    void* out;       // [T][ld] of `type`: this piece's columns
    int64_t T, ld;
    int v0, width;   // first column of the piece in the vocabulary, columns of the piece
    float c;         // log2(e) / tau
    float up;        // power of two that keeps small probabilities above the smallest fp16 (1 for bf16)
    int type;
  };
  static __device__ __forceinline__ void tile(const Args& a, const Tile& t, uint32_t tmem, int row_block, int e, int lane,
                                              char* staging) {
    const int row0 = row_block * iwp_tc::TILE_M + (e % 4) * 32, row = row0 + lane;
    const int col0 = t.n * iwp_tc::TILE_N + (e / 4) * (iwp_tc::TILE_N / 2);
    int pos = 0, next = NO_COLUMN;
    float scale = 0.f, lse2 = 0.f;
    if (row < a.T) {
      scale = a.en.row_scale[row] * a.up;
      lse2 = a.lse[row] * LOG2E;
      if (scale != 0.f) {
        pos = first_entry(a.en, a.T, row, a.v0 + col0);
        if (pos < a.en.k) next = a.en.column[pos * a.T + row];
      }
    }
#pragma unroll 1
    for (int c0 = col0; c0 < min(col0 + iwp_tc::TILE_N / 2, a.width); c0 += 32) {
      float v[32];
      iwp_tc::tmem_load32(tmem + (c0 - col0), v);
      // a row that gives nothing writes zeros whatever its logits are
#pragma unroll
      for (int j = 0; j < 32; j++) v[j] = scale == 0.f ? 0.f : exp2f(fmaf(v[j], a.c, -lse2));
      const int end = a.v0 + c0 + 32;
      if (__any_sync(0xFFFFFFFFu, next < end)) {
        float* mine = reinterpret_cast<float*>(staging + lane * iwp_tc::STAGING_PITCH);
#pragma unroll
        for (int j = 0; j < 32; j += 4) *reinterpret_cast<float4*>(mine + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
        while (next < end) {
          mine[next - (a.v0 + c0)] -= a.en.q[pos * a.T + row];
          pos++;
          next = pos < a.en.k ? a.en.column[pos * a.T + row] : NO_COLUMN;
        }
#pragma unroll
        for (int j = 0; j < 32; j += 4) {
          const float4 x = *reinterpret_cast<const float4*>(mine + j);
          v[j] = x.x, v[j + 1] = x.y, v[j + 2] = x.z, v[j + 3] = x.w;
        }
        __syncwarp();
      }
#pragma unroll
      for (int j = 0; j < 32; j++) v[j] *= scale;
      iwp_tc::store_chunk(v, staging, a.out, a.ld, a.type, true, false, row0, static_cast<int>(a.T), c0, a.width, lane);
    }
  }
};

// ---- epilogue of the gradient products ------------------------------------------------------------------

// What both gradients are multiplied with: `factor` (scale * tau / up) * gmax * dloss / n.
struct Factor {
  const Header* hdr;
  const float* dloss;
  float factor;
  int mean, by_rows;
  __device__ __forceinline__ float get() const {
    float f = factor;
    if (by_rows) f *= hdr->gmax;
    if (dloss) f *= *dloss;
    if (mean) f /= static_cast<float>(max(hdr->n_rows, 1));
    return f;
  }
};

struct Out {
  struct Args {
    Factor f;
    void* out;
    int64_t ld, split_stride;  // elements
    int rows, cols, type, wide, add, raw;  // raw: partial sums, the factor is applied later
  };
  static __device__ __forceinline__ void tile(const Args& a, const Tile& t, uint32_t tmem, int row_block, int e, int lane,
                                              char* staging) {
    const int row0 = row_block * iwp_tc::TILE_M + (e % 4) * 32;
    const int col0 = t.n * iwp_tc::TILE_N + (e / 4) * (iwp_tc::TILE_N / 2);
    const float f = a.raw ? 1.f : a.f.get();
    char* const out = static_cast<char*>(a.out) + t.split * a.split_stride * (a.type == IWP_F32 ? 4 : 2);
#pragma unroll 1
    for (int c0 = col0; c0 < min(col0 + iwp_tc::TILE_N / 2, a.cols); c0 += 32) {
      float v[32];
      iwp_tc::tmem_load32(tmem + (c0 - col0), v);
#pragma unroll
      for (int j = 0; j < 32; j++) v[j] *= f;
      iwp_tc::store_chunk(v, staging, out, a.ld, a.type, a.wide, a.add, row0, a.rows, c0, a.cols, lane);
    }
  }
};

// dhidden = factor * sum over the splits (in order), rounded once.
__global__ void k_join(Factor f, const float* part, int splits, int64_t rows, int cols, void* out, int64_t ld, int type, int add) {
  const float k = f.get();
  const int64_t n = rows * cols;
  for (int64_t i = blockIdx.x * int64_t(blockDim.x) + threadIdx.x; i < n; i += int64_t(gridDim.x) * blockDim.x) {
    float x = 0.f;
    for (int s = 0; s < splits; s++) x += part[s * n + i];
    x *= k;
    const int64_t at = (i / cols) * ld + i % cols;
    if (add) x += iwp_tc::load_as_float(out, at, type);
    iwp_tc::store_as(out, at, x, type);
  }
}

// ---- targets -> entries -----------------------------------------------------------------------------------

__global__ void k_hard_targets(Header* hdr, Entries en, const int64_t* targets, int64_t ignore, int64_t T, int64_t V) {
  const int64_t t = blockIdx.x * int64_t(blockDim.x) + threadIdx.x;
  bool has = false;
  if (t < T) {
    const int64_t y = targets[t];
    const bool ignored = y == ignore, good = !ignored && y >= 0 && y < V;
    en.column[t] = good ? static_cast<int>(y) : NO_COLUMN;
    en.q[t] = good ? 1.f : 0.f;
    en.const_term[t] = ignored || good ? 0.f : CUDART_NAN_F;
    en.row_scale[t] = good ? 1.f : 0.f;
    if (!ignored && !good) atomicExch(&hdr->status, IWP_ERR_INVALID);
    has = !ignored;
  }
  const unsigned b = __ballot_sync(0xFFFFFFFFu, has);
  if ((threadIdx.x & 31) == 0 && b) atomicAdd(&hdr->n_rows, __popc(b));
}

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

// One warp per row: softmax over the row's teacher logits, entries ordered by column (by counting the smaller ones).
__global__ void k_soft_targets(Header* hdr, Entries en, const void* ids, int64_t ids_ld, int ids_bytes, const void* logits,
                               int64_t logits_ld, int type, float inv_tau, int64_t T, int64_t V) {
  extern __shared__ int sh_col[];
  const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, K = en.k;
  const int64_t t = blockIdx.x * int64_t(warps) + warp;
  if (t >= T) return;
  int* col = sh_col + warp * K;
  float top = -CUDART_INF_F;
  bool bad = false, nan = false;
  for (int k = lane; k < K; k += 32) {
    const int64_t id = load_id(ids, t * ids_ld + k, ids_bytes);
    const float x = iwp_tc::load_as_float(logits, t * logits_ld + k, type) * inv_tau;
    bad |= id >= V;
    const bool used = id >= 0 && id < V && x != -CUDART_INF_F;  // NaN takes part
    col[k] = used ? static_cast<int>(id) : NO_COLUMN;
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
    if (col[k] != NO_COLUMN) sum += expf(iwp_tc::load_as_float(logits, t * logits_ld + k, type) * inv_tau - top);
  sum = warp_sum(sum);
  const bool has = top != -CUDART_INF_F || nan;
  const float log_sum = logf(sum);
  float term = 0.f;
  for (int k = lane; k < K; k += 32) {
    const int c = col[k];
    int rank = 0;
    for (int j = 0; j < K; j++) rank += col[j] < c || (col[j] == c && j < k);
    float q = 0.f;
    if (c != NO_COLUMN) {
      const float lq = iwp_tc::load_as_float(logits, t * logits_ld + k, type) * inv_tau - top - log_sum;
      q = expf(lq);
      if (q != 0.f) term += q * lq;
    }
    en.column[rank * T + t] = bad ? NO_COLUMN : c;
    en.q[rank * T + t] = q;
  }
  term = warp_sum(term);
  if (lane == 0) {
    en.const_term[t] = bad ? CUDART_NAN_F : has ? term : 0.f;
    en.row_scale[t] = has && !bad ? 1.f : 0.f;
    if (bad) atomicExch(&hdr->status, IWP_ERR_INVALID);
    if (has || bad) atomicAdd(&hdr->n_rows, 1);
  }
}

// ---- per-row upstream gradients: their largest magnitude, and the rows relative to it ------------------------

__global__ void k_row_scales(Header* hdr, float* row_scale, const float* dloss_rows, int64_t T) {
  __shared__ float sh[32];
  float m = 0.f;
  for (int64_t t = threadIdx.x; t < T; t += blockDim.x)
    if (row_scale[t] != 0.f) m = fmaxf(m, fabsf(dloss_rows[t]));
  m = warp_max(m);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = m;
  __syncthreads();
  m = warp_max((threadIdx.x & 31) < (blockDim.x >> 5) ? sh[threadIdx.x & 31] : 0.f);
  if (threadIdx.x == 0) hdr->gmax = m;
  for (int64_t t = threadIdx.x; t < T; t += blockDim.x)
    if (row_scale[t] != 0.f) row_scale[t] = m > 0.f ? dloss_rows[t] / m : dloss_rows[t];
}

// ---- finish of the forward pass --------------------------------------------------------------------------

// Blocks of 32 warps take 32 rows (lane = row): each warp joins every 32nd part, the first warp joins the warps.
// The last block to finish adds the blocks' sums in order.
__global__ void __launch_bounds__(1024) k_finish(Header* hdr, Entries en, const float2* part, int parts, const float* z_at, float tau,
                                                 int64_t T, float* rows, float* lse, float* loss, int mean, float* block_sum) {
  __shared__ float2 sh[32][33];
  __shared__ bool last;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t row = blockIdx.x * 32ll + lane;
  float m = -CUDART_INF_F, s = 0.f;
  if (row < T) {
#pragma unroll 4
    for (int p = warp; p < parts; p += 32) {
      const float2 x = part[p * T + row];
      const float mn = fmaxf(m, x.x), ref = mn == -CUDART_INF_F ? 0.f : mn;
      s = s * exp2f(m - ref) + x.y * exp2f(x.x - ref);
      m = mn;
    }
  }
  sh[warp][lane] = make_float2(m, s);
  __syncthreads();
  if (warp == 0) {
    float r = 0.f;
    if (row < T) {
      for (int w = 1; w < 32; w++) {
        const float2 x = sh[w][lane];
        const float mn = fmaxf(m, x.x), ref = mn == -CUDART_INF_F ? 0.f : mn;
        s = s * exp2f(m - ref) + x.y * exp2f(x.x - ref);
        m = mn;
      }
      const float l = (m + log2f(s)) * LN2;
      lse[row] = l;
      if (rows || loss) {
        // sum of q (z / tau) in units of the row's lse, so that a confident row keeps its small loss
        const float c = en.const_term[row];
        float below = 0.f;
        if (en.row_scale[row] != 0.f || c != 0.f) {
          for (int k = 0; k < en.k; k++) {
            if (en.column[k * T + row] == NO_COLUMN) break;
            const float q = en.q[k * T + row];
            if (q != 0.f) below += q * (l - z_at[k * T + row] / tau);
          }
          r = tau * tau * (c + below);
        }
        if (rows) rows[row] = r;
      }
    }
    r = warp_sum(r);
    if (lane == 0) {
      block_sum[blockIdx.x] = r;
      __threadfence();
      last = atomicAdd(&hdr->ticket, 1u) == gridDim.x - 1;
    }
  }
  __syncthreads();
  if (last && loss) {
    __threadfence();
    float x = 0.f;
    for (int b = threadIdx.x; b < static_cast<int>(gridDim.x); b += 1024) x += __ldcg(block_sum + b);
    x = warp_sum(x);
    __shared__ float sums[32];
    if (lane == 0) sums[warp] = x;
    __syncthreads();
    if (warp == 0) {
      x = warp_sum(sums[lane]);
      const int n = hdr->n_rows;
      if (lane == 0) *loss = n == 0 ? 0.f : mean ? x / static_cast<float>(n) : x;
    }
  }
}

// Rows of `cols` 16-bit elements to rows of `ld_to` (a multiple of 8), for operands TMA cannot address.
__global__ void k_align_rows(const uint16_t* from, int64_t ld_from, uint16_t* to, int64_t ld_to, int64_t rows, int cols) {
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
    for (int c = threadIdx.x; c < cols; c += blockDim.x) to[r * ld_to + c] = from[r * ld_from + c];
}

}  // namespace iwp_head
