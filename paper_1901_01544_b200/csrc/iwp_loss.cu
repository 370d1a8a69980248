// iwp_loss.cu - C entries of the losses (include/iwp_loss.h): argument checks, workspace layout, launches.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>
#include <type_traits>
#include <utility>

#include "iwp_balance.cuh"
#include "iwp_head.cuh"
#include "iwp_host.hpp"

namespace {

using namespace iwp_host;

constexpr int64_t ROOM = 0xFFFF;                 // how far 32-bit positions may run beyond a size
constexpr int64_t MAX_SIZE = 0x7FFFFFFF - ROOM;  // of tokens, vocabulary, width and strides
constexpr int64_t MAX_ELEMENTS = int64_t(1) << 46;
constexpr int64_t LEAST_PIECE = int64_t(1) << 30;
constexpr int FEW_TILES = 296;           // four per CTA pair: above this a product takes its widest tiles
constexpr int FEW_BLOCKS = 296;           // of the pass over a few tokens: two per SM
static_assert(2 * iwp_tc::TILE_N <= ROOM && iwp_head::FACTOR_COLUMNS + iwp_tc::TILE_N <= ROOM &&
                  FEW_BLOCKS * (iwp_head::FEW_THREADS / 32) * iwp_head::FEW_ROWS + iwp_tc::TILE_N <= ROOM,
              "positions of the kernels' last steps stay within 32 bits");
constexpr int64_t FEW_ELEMENTS = 32768;   // of hidden states, which stay in 64 KB of shared memory
constexpr int64_t JOIN_TILES = 2 * 148;  // a split dhidden has at most this many partial tiles

// cuTensorMapEncodeTiled through the runtime, so that the library links against no driver stub.
using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                            const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

Encode encoder() {
  static Encode fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q{};
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      p = nullptr;
    }
    return reinterpret_cast<Encode>(p);
  }();
  return fn;
}

// A row-major matrix of 16-bit elements, copied in boxes of box_rows rows and 64 elements (128 bytes, swizzled).
// Elements outside read as zero.
bool make_map(CUtensorMap* map, const void* p, int64_t rows, int64_t cols, int64_t ld, int box_rows, int dtype) {
  Encode enc = encoder();
  if (!enc) return false;
  cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
  cuuint64_t strides[1] = {static_cast<cuuint64_t>(ld) * 2};
  cuuint32_t box[2] = {64, static_cast<cuuint32_t>(box_rows)}, step[2] = {1, 1};
  return enc(map, dtype == IWP_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void*>(p), dims,
             strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr int SEGMENT = 1024 / iwp_tc::BLOCK_K;  // most blocks of K that are summed in tensor memory

// How many CTA pairs of a product kernel the device holds at once: the persistent grid (a pair that had to wait for
// another to end would double the time).  Looked up once per device, with the kernel's shared memory limit.
template <class Kernel>
int resident_pairs(Kernel kernel, int smem, std::atomic<int>* cached) {
  const int dev = device();
  if (dev < 0) return 0;
  if (cached[dev]) return cached[dev];
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return 0;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(iwp_tc::CG);
  cfg.blockDim = dim3(iwp_tc::THREADS);
  cfg.dynamicSmemBytes = static_cast<size_t>(smem);
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = iwp_tc::CG;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) return 0;
  cached[dev] = n;
  return n;
}

struct Matrix {
  const void* p;
  int64_t rows, cols, ld;
};

struct Shape {
  int64_t m, n, k;
  int64_t m_tiles() const { return tiles_of(m, iwp_tc::CG * iwp_tc::TILE_M); }
  int64_t k_blocks() const { return tiles_of(k, iwp_tc::BLOCK_K); }
  int64_t tiles(int n_cols) const { return m_tiles() * tiles_of(n, n_cols); }
  // clocks of a tile with its K in `splits` parts, about: per block of K the products or the loads, whichever takes
  // longer (32, 24 or 20 KB per CTA; more where the other operand is streamed for this one row of tiles), but no less
  // than an epilogue
  double clocks(int n_cols, int splits) const {
    const double block = n_cols == 256 ? (m_tiles() == 1 ? 680 : 520) : n_cols == 128 ? 385 : 320;
    const double products = static_cast<double>(tiles_of(k_blocks(), splits)) * block, epilogue = 700 + 11.0 * n_cols;
    return (products > epilogue ? products : epilogue) + 300;
  }
};

// Width of a single product's tiles: 256 where there are tiles enough for all pairs, less where the narrower tiles'
// shorter time wins over their poorer use of the loads.  (256 x 1000 x 2048, all of a training pass: 32.5 us with narrow
// tiles, 36.9 with 256; 40 x 8192 x 512: 32.0 and 33.2; from a few hundred wide tiles on there is no difference.)
int pick_tile_n(const Shape& s, int pairs) {
  if (s.tiles(256) > FEW_TILES) return 256;
  int best = 256;
  double least = 0;
  for (int n : {256, 128, 64}) {
    const double time = static_cast<double>(tiles_of(s.tiles(n), pairs)) * s.clocks(n, 1);
    if (n == 256 || time < 0.95 * least) best = n, least = time;
  }
  return best;
}

// Plan of the two gradient products of a piece in one launch: the width of the tiles, the number of parts of dhidden's
// K (the vocabulary), and how its tiles and dweight's are dealt to the pairs (Problems).
struct Deal {
  int tile_n, splits, rounds, rest, fill;
};

Deal deal_gradients(const Shape* dh, const Shape* dw, int pairs, int fixed_splits) {
  Deal best{256, 1, 0, 0, 0};
  double least = -1;
  for (int n : {256, 128, 64}) {
    const int64_t one = dh ? dh->tiles(n) : 0, w = dw ? dw->tiles(n) : 0;
    if (n < 256 && one + w > FEW_TILES) break;
    int64_t most = dh ? dh->k_blocks() / 4 : 1;
    if (dh && most > JOIN_TILES / one) most = JOIN_TILES / one;
    if (most < 1) most = 1;
    for (int64_t s = fixed_splits ? fixed_splits : 1; s <= (fixed_splits ? fixed_splits : most); s++) {
      const double ch = dh ? dh->clocks(n, static_cast<int>(s)) : 0, cw = dw ? dw->clocks(n, 1) : 1;
      const int64_t tiles = one * s;
      Deal d{n, static_cast<int>(s), static_cast<int>(tiles / pairs), static_cast<int>(tiles % pairs), 0};
      // pairs with one more tile of dhidden end at `long_way`, the others at `short_way`; what is left of dweight goes to
      // the others first
      int64_t left = w;
      const int64_t others = pairs - d.rest;
      double long_way = d.rest ? ch : 0, short_way = 0;
      if (d.rest) {
        int64_t fill = static_cast<int64_t>(ch / cw);
        if (fill > w / others) fill = w / others;
        d.fill = static_cast<int>(fill);
        left -= fill * others;
        short_way = static_cast<double>(fill) * cw;
      }
      short_way += static_cast<double>(tiles_of(left, pairs)) * cw;
      if (left > others && d.rest) long_way += static_cast<double>(tiles_of(left - others, pairs)) * cw;
      double time = d.rounds * ch + (long_way > short_way ? long_way : short_way);
      // parts are joined by a launch of its own: its start, and each part written and read once at about 2500 bytes per clock
      if (s > 1) time += 15000 + static_cast<double>(dh->m) * static_cast<double>(dh->n) * 8 * static_cast<double>(s) / 2500;
      if (least < 0 || time < least) least = time, best = d;
    }
  }
  return best;
}

// C[M, N] = A B^T: a K-contiguous operand is [M or N][K], the other [K][M or N].
bool make_problem(iwp_tc::Problem* q, const Matrix& A, bool a_kc, const Matrix& B, bool b_kc, int dtype, int tile_n, int splits) {
  const Shape s{a_kc ? A.rows : A.cols, b_kc ? B.rows : B.cols, a_kc ? A.cols : A.rows};
  if (!make_map(&q->a, A.p, A.rows, A.cols, A.ld, a_kc ? iwp_tc::TILE_M : iwp_tc::BLOCK_K, dtype) ||
      !make_map(&q->b, B.p, B.rows, B.cols, B.ld, b_kc ? tile_n / iwp_tc::CG : iwp_tc::BLOCK_K, dtype))
    return false;
  q->m_tiles = static_cast<int>(s.m_tiles());
  q->n_tiles = static_cast<int>(tiles_of(s.n, tile_n));
  q->tile_n = tile_n;
  q->k_blocks = static_cast<int>(s.k_blocks());
  q->splits = splits;
  const int64_t part = tiles_of(s.k_blocks(), splits);
  q->seg = static_cast<int>(tiles_of(part, tiles_of(part, SEGMENT)));  // of even length
  // f32 accumulator; operand types; which operands are M/N-contiguous; N / 8; M / 16
  const uint32_t type = dtype == IWP_BF16 ? 1u : 0u;
  q->use_other = nullptr;
  q->idesc = (1u << 4) | (type << 7) | (type << 10) | ((a_kc ? 0u : 1u) << 15) | ((b_kc ? 0u : 1u) << 16) |
             (static_cast<uint32_t>(tile_n / 8) << 17) | ((iwp_tc::TILE_M * iwp_tc::CG / 16u) << 24);
  q->a_kc = a_kc;
  q->b_kc = b_kc;
  return true;
}

int64_t segments(const iwp_tc::Problem& q) { return q.splits ? tiles_of(tiles_of(q.k_blocks, q.splits), q.seg) : 0; }

template <class Epi, int N>
int pairs_of() {
  static std::atomic<int> cached[MAX_DEVICES] = {};
  return resident_pairs(iwp_tc::k_product<N, Epi>, iwp_tc::smem_bytes(Epi::AREAS), cached);
}

template <class Epi, int N>
int launch_product(iwp_tc::Problems<N>& w, const typename Epi::Args& args, int pairs, cudaStream_t st) {
  int64_t total = 0;
  for (const auto& q : w.p) total += int64_t(q.m_tiles) * q.n_tiles * q.splits;
  if (total > MAX_SIZE) return IWP_ERR_INVALID;
  const int tile_n = w.p[N - 1].n_tiles ? w.p[N - 1].tile_n : w.p[0].tile_n;  // the same for both
  w.b_bytes = static_cast<int>(up_to(tile_n / iwp_tc::CG, 64)) * iwp_tc::BLOCK_K * 2;
  w.stages = iwp_tc::ring_bytes(Epi::AREAS) / (iwp_tc::A_BYTES + w.b_bytes);
  if (w.stages > iwp_tc::MAX_STAGES) w.stages = iwp_tc::MAX_STAGES;
  LOSS_CUDA(launch(iwp_tc::k_product<N, Epi>, iwp_tc::CG * (total < pairs ? total : pairs), iwp_tc::THREADS, iwp_tc::smem_bytes(Epi::AREAS),
                   iwp_tc::CG, st, w, args));
  return IWP_OK;
}

// ---- output head ----------------------------------------------------------------------------------------

struct HeadPlan {
  bool grad, few, pack_hidden, pack_weight;
  bool split_rows;  // fp16 with an upstream gradient per row: k_row_scales
  int64_t k, piece, pieces, d_pad;
  // offsets into the workspace
  int64_t column, q, const_term, row_scale, row_power, rows, z_at, part, hidden, weight, copy, probs, join, bytes;
};

bool needs_copy(const void* p, int64_t ld) { return !aligned(p, 16) || ld % 8 != 0; }

bool head_args_ok(const iwp_head_args* a) {
  if (!a || a->tokens < 0 || a->tokens > MAX_SIZE || a->vocab < 1 || a->vocab > MAX_SIZE || a->dim < 1 || a->dim > MAX_SIZE) return false;
  // (what no device could hold, so that sizes in bytes stay far from the end of 64 bits)
  if (a->tokens * a->vocab > MAX_ELEMENTS || a->tokens * a->dim > MAX_ELEMENTS || a->vocab * a->dim > MAX_ELEMENTS) return false;
  if (a->dtype != IWP_BF16 && a->dtype != IWP_F16) return false;
  if (!a->targets && (a->top_k < 1 || a->top_k > iwp_head::MAX_TOP)) return false;
  if (a->hidden_ld < a->dim || a->weight_ld < a->dim || a->hidden_ld > MAX_SIZE || a->weight_ld > MAX_SIZE) return false;
  if (a->dhidden && (a->dhidden_ld < a->dim || (a->dhidden_type != a->dtype && a->dhidden_type != IWP_F32))) return false;
  if (a->dweight && (a->dweight_ld < a->dim || (a->dweight_type != a->dtype && a->dweight_type != IWP_F32))) return false;
  return a->piece_bytes >= 0;
}

HeadPlan head_plan(const iwp_head_args* a) {
  HeadPlan p{};
  const int64_t T = a->tokens, V = a->vocab, D = a->dim;
  p.grad = a->dhidden || a->dweight;
  p.k = a->targets ? 1 : a->top_k;
  p.d_pad = up_to(D, 8);
  p.pack_hidden = needs_copy(a->hidden, a->hidden_ld);
  p.pack_weight = needs_copy(a->weight, a->weight_ld);
  p.few = !p.grad && T <= iwp_head::FEW_TOKENS && T * up_to(D, 8) <= FEW_ELEMENTS && (D % 8 == 0 || (p.pack_hidden && p.pack_weight));
  int64_t at = IWP_LOSS_STATE;
  auto take = [&at](int64_t n) {
    const int64_t o = at;
    at += up_to(n, 256);
    return o;
  };
  if (!a->targets) {
    p.column = take(4 * p.k * T);
    p.q = take(4 * p.k * T);
    p.const_term = take(4 * T);
  }
  p.split_rows = p.grad && a->dloss_rows && a->dtype == IWP_F16;
  if (p.split_rows) {
    p.row_scale = take(4 * T);
    p.row_power = take(4 * T);
  }
  if (a->dweight) p.copy = take(2 * T * p.d_pad);
  p.rows = take(4 * T);
  if (!a->have_lse) {
    p.z_at = take(4 * p.k * T);
    // a part is half a tile of at least 64 columns; narrow tiles are taken where those of 256 columns would be few
    // (FEW_TILES), i.e. at most 8 parts of 8 bytes for each of a tile's 256 rows
    const int64_t wide = 8 * T * 2 * tiles_of(V, 256) + 8 * iwp_head::FEW_TOKENS * FEW_BLOCKS, narrow = 8 * T * 2 * tiles_of(V, 64), most = int64_t(FEW_TILES) * 256 * 64;
    p.part = take(wide > most ? wide : narrow < most ? narrow : most);
  }
  if (p.pack_hidden) p.hidden = take(2 * T * p.d_pad);
  if (p.pack_weight) p.weight = take(2 * V * p.d_pad);
  if (p.grad) {
    // By default no more than the weights and their gradient take: 8192 tokens x 131072 x 4096 then stay one piece (2 GiB)
    // and run in 23.1 ms, against 24.8 in two pieces of 1 GiB, the logits of one of which are computed twice.
    const int64_t own = 4 * V * D;
    const int64_t limit = a->piece_bytes ? a->piece_bytes : own > LEAST_PIECE ? own : LEAST_PIECE;
    const int64_t v_pad = up_to(V, iwp_tc::TILE_N), t = T > 0 ? T : 1;
    int64_t width = limit / (2 * t) / iwp_tc::TILE_N * iwp_tc::TILE_N;
    if (width < iwp_tc::TILE_N) width = iwp_tc::TILE_N;
    if (width > v_pad) width = v_pad;
    p.pieces = tiles_of(v_pad, width);
    p.piece = up_to(tiles_of(v_pad, p.pieces), iwp_tc::TILE_N);
    p.pieces = tiles_of(v_pad, p.piece);
    const int64_t most = 2 * t * v_pad < limit ? 2 * t * v_pad : limit, least = 2 * t * iwp_tc::TILE_N;
    p.probs = take(most > least ? most : least);
  }
  if (a->dhidden) {
    const int64_t one = 4 * T * up_to(D, 4), split = JOIN_TILES * 4 * iwp_tc::CG * iwp_tc::TILE_M * iwp_tc::TILE_N;
    p.join = take(one > split ? one : split);
  }
  p.bytes = at;
  return p;
}

int head_run(const iwp_head_args* a, const HeadPlan& p, cudaStream_t st) {
  namespace H = iwp_head;
  const int64_t T = a->tokens, V = a->vocab, D = a->dim;
  char* const ws = static_cast<char*>(a->workspace);
  auto* hdr = static_cast<H::Header*>(a->state ? a->state : a->workspace);
  // one persistent grid for all products (the deal of the gradients counts on it)
  const int pairs = std::min({pairs_of<H::Logits<H::NO_CODES>, 1>(), pairs_of<H::Logits<H::HALF_CODES>, 1>(), pairs_of<H::Logits<H::LOG_CODES>, 1>(),
                              pairs_of<H::Probs, 1>(), pairs_of<H::Out<false>, 2>(), pairs_of<H::Out<true>, 2>()});
  if (pairs < 1) {
    cudaGetLastError();
    return IWP_ERR_CUDA;
  }
  const int sms = 2 * pairs;
  const float tau = a->targets ? 1.f : a->temperature, c = H::LOG2E / tau;
  if (T == 0) {
    if (a->loss && !a->have_lse) LOSS_CUDA(cudaMemsetAsync(a->loss, 0, 4, st));
    if (a->dweight && !a->accumulate) {
      const int64_t e = a->dweight_type == IWP_F32 ? 4 : 2;
      LOSS_CUDA(cudaMemset2DAsync(a->dweight, a->dweight_ld * e, 0, D * e, V, st));
    }
    return IWP_OK;
  }
  H::Targets en{};
  en.hard = a->targets;
  en.ignore = a->ignore_index;
  en.V = static_cast<int>(V);
  en.k = static_cast<int>(p.k);
  if (!a->targets) {
    int* const column = reinterpret_cast<int*>(ws + p.column);
    float* const q = reinterpret_cast<float*>(ws + p.q);
    float* const term = reinterpret_cast<float*>(ws + p.const_term);
    LOSS_CUDA(launch(H::k_soft_targets, tiles_of(T, 4), 128, 4 * 8 * p.k, 1, st, column, q, term, a->top_ids, a->top_ids_ld, a->ids_bytes,
                     a->top_logits, a->top_logits_ld, a->top_type, en.k, 1.f / tau, T, V));
    en.column = column;
    en.q = q;
    en.const_term = term;
  }
  float* const row_scale = reinterpret_cast<float*>(ws + p.row_scale);
  float* const row_power = p.split_rows ? reinterpret_cast<float*>(ws + p.row_power) : nullptr;
  if (p.split_rows) LOSS_CUDA(launch(H::k_row_scales, 1, 1024, 0, 1, st, hdr, en, row_scale, row_power, a->dloss_rows, T));
  if (p.grad) en.scale = p.split_rows ? row_scale : a->dloss_rows;
  Matrix h{a->hidden, T, D, a->hidden_ld}, w{a->weight, V, D, a->weight_ld};
  auto align_rows = [&](Matrix& m, int64_t at) {
    const int64_t warps = tiles_of(m.rows, 8), blocks = warps < 8 * sms ? warps : 8 * sms;
    const auto kernel = aligned(m.p, 8) && m.ld % 4 == 0   ? H::k_align_rows<uint2>
                        : aligned(m.p, 4) && m.ld % 2 == 0 ? H::k_align_rows<uint32_t>
                                                           : H::k_align_rows<uint16_t>;
    const cudaError_t e = launch(kernel, blocks, 256, 0, 1, st, static_cast<const uint16_t*>(m.p), m.ld, reinterpret_cast<uint16_t*>(ws + at), p.d_pad,
                                 m.rows, static_cast<int>(D));
    m.p = ws + at, m.ld = p.d_pad;
    return e;
  };
  if (p.pack_hidden) LOSS_CUDA(align_rows(h, p.hidden));
  if (p.pack_weight) LOSS_CUDA(align_rows(w, p.weight));
  // dweight's product: the hidden states; with the rows' scales; or, if the device finds that they have to be, clean
  const Matrix h_copy{ws + p.copy, T, D, p.d_pad}, h_dw = p.split_rows ? h_copy : h;
  const bool may_clean = a->dweight && !p.split_rows;
  const H::Clean copy{static_cast<const uint16_t*>(h.p), may_clean ? reinterpret_cast<uint16_t*>(ws + p.copy) : nullptr, h.ld, p.d_pad, T,
                      static_cast<int>(D)};
  if (a->have_lse) LOSS_CUDA(launch(H::k_count_rows, 1, 1024, 0, 1, st, hdr, en, a->lse, copy, T));
  if (p.split_rows && a->dweight) {
    const int64_t blocks = tiles_of(T, 8);
    LOSS_CUDA(launch(H::k_scaled_rows, blocks < 8 * sms ? blocks : 8 * sms, 256, 0, 1, st, hdr, row_scale, row_power, static_cast<const __half*>(h.p),
                     h.ld, reinterpret_cast<__half*>(ws + p.copy), p.d_pad, T, static_cast<int>(D)));
  }

  const float up = a->dtype == IWP_F16 ? 8192.f : 1.f;
  uint16_t* const probs = reinterpret_cast<uint16_t*>(ws + p.probs);
  const int64_t kept = p.grad && !a->have_lse ? p.pieces - 1 : -1;  // the piece whose codes the logits pass leaves behind
  if (!a->have_lse) {
    H::Rows ra{};
    ra.hdr = hdr;
    ra.en = en;
    ra.part = reinterpret_cast<float2*>(ws + p.part);
    ra.z_at = reinterpret_cast<float*>(ws + p.z_at);
    ra.rows = a->rows ? a->rows : reinterpret_cast<float*>(ws + p.rows);
    ra.lse = a->lse;
    ra.loss = a->loss;
    ra.T = T;
    ra.mean = a->mean;
    ra.tau = tau;
    ra.c = c;
    ra.lanes = T <= 8 * sms ? H::ROW_THREADS : 32;  // a block per row while all blocks run at once, a warp after that
    const int64_t row_blocks = ra.lanes == 32 ? tiles_of(T, H::ROW_THREADS / 32) : T;
    if (p.few) {
      H::Few fa{};
      fa.en = en;
      fa.hidden = h.p;
      fa.weight = w.p;
      fa.part = reinterpret_cast<float2*>(ws + p.part);
      fa.z_at = reinterpret_cast<float*>(ws + p.z_at);
      fa.hidden_ld = h.ld;
      fa.weight_ld = w.ld;
      fa.T = static_cast<int>(T);
      fa.V = static_cast<int>(V);
      fa.D = static_cast<int>(D);
      fa.type = a->dtype;
      fa.c = c;
      constexpr int warps = H::FEW_THREADS / 32;
      const int64_t whole = tiles_of(V, warps * H::FEW_ROWS);
      fa.blocks = static_cast<int>(whole < FEW_BLOCKS ? whole : FEW_BLOCKS);
      const int64_t grid = fa.blocks + tiles_of(T * p.k, warps);
      auto few = [&](auto tokens) {
        constexpr int N = decltype(tokens)::value;
        auto kernel = H::k_few_tokens<N>;
        static std::atomic<bool> ready[MAX_DEVICES] = {};
        const int dev = device();
        if (dev < 0) return cudaErrorInvalidDevice;
        if (!ready[dev]) {
          const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(2 * FEW_ELEMENTS));
          if (e != cudaSuccess) return e;
          ready[dev] = true;
        }
        return launch(kernel, grid, H::FEW_THREADS, static_cast<size_t>(16 * N * tiles_of(D, 8)), 1, st, fa);
      };
      LOSS_CUDA(T == 1 ? few(std::integral_constant<int, 1>{}) : few(std::integral_constant<int, 2>{}));
      ra.parts = fa.blocks;
      LOSS_CUDA(launch(H::k_rows, row_blocks, H::ROW_THREADS, 0, 1, st, ra));
      return IWP_OK;
    }
    const Shape shape{T, V, D};
    const int tile_n = pick_tile_n(shape, pairs);
    iwp_tc::Problems<1> work;
    if (!make_problem(&work.p[0], h, true, w, true, a->dtype, tile_n, 1)) return IWP_ERR_CUDA;
    work.status = &hdr->status;
    work.early = !a->targets && !p.split_rows && !p.pack_hidden && !p.pack_weight;  // k_soft_targets comes right before
    const int parts = 2 * work.p[0].n_tiles;
    const int64_t v0 = kept >= 0 ? kept * p.piece : 0;
    auto logits = [&](auto epilogue) {
      using Epi = decltype(epilogue);
      typename Epi::Args la{};
      la.en = en;
      la.T = T;
      la.V = static_cast<int>(V);
      la.c = c;
      la.part = reinterpret_cast<float2*>(ws + p.part);
      la.parts = parts;
      la.z_at = reinterpret_cast<float*>(ws + p.z_at);
      la.codes = probs;
      la.ld = p.piece;
      la.v0 = static_cast<int>(v0);
      la.width = static_cast<int>(p.piece);
      if (kept >= 0 && !make_map(&la.map, probs, T, p.piece, p.piece, 32, a->dtype)) return static_cast<int>(IWP_ERR_CUDA);
      return launch_product<Epi, 1>(work, la, pairs, st);
    };
    const int failed = kept < 0 ? logits(H::Logits<H::NO_CODES>{}) : a->dtype == IWP_F16 ? logits(H::Logits<H::LOG_CODES>{}) : logits(H::Logits<H::HALF_CODES>{});
    if (failed) return failed;
    ra.parts = parts;
    LOSS_CUDA(launch(H::k_rows, row_blocks, H::ROW_THREADS, 0, 1, st, ra));
    if (kept >= 0) {
      H::Factors fa{};
      fa.en = en;
      fa.part = ra.part;
      fa.z_at = ra.z_at;
      fa.lse = a->lse;
      fa.codes = probs;
      fa.ld = p.piece;
      fa.parts = parts;
      fa.part_shift = tile_n == 256 ? 7 : tile_n == 128 ? 6 : 5;
      fa.v0 = static_cast<int>(v0);
      fa.width = static_cast<int>(V - fa.v0 < p.piece ? V - fa.v0 : p.piece);
      fa.chunks = static_cast<int>(tiles_of(fa.width, H::FACTOR_COLUMNS));
      fa.log_codes = a->dtype == IWP_F16;
      fa.c = c;
      fa.up = up;
      fa.hdr = hdr;
      fa.blocks = T * fa.chunks;
      fa.copy = copy;
      const int64_t others = may_clean ? std::min<int64_t>(tiles_of(T, H::FACTOR_THREADS / 32), sms) : 0;
      if (fa.blocks + others > MAX_SIZE) return IWP_ERR_INVALID;
      LOSS_CUDA(launch(H::k_factors, fa.blocks + others, H::FACTOR_THREADS, 0, 1, st, fa));
    }
  }
  if (!p.grad) return IWP_OK;

  H::OutArgs oa{};
  oa.f.hdr = hdr;
  oa.f.dloss = a->dloss;
  oa.f.factor = a->scale * tau / up;
  oa.f.mean = a->mean;
  oa.m[0].row_power = row_power;
  oa.m[1].by_gmax = p.split_rows;
  auto copy_map = [](H::OutMatrix& o) {
    o.by_copy = o.type != IWP_F32 && o.wide && !o.add;
    return !o.by_copy || make_map(&o.map, o.out, o.rows, o.cols, o.ld, 32, o.type);
  };
  int splits = 1;
  for (int64_t done = 0; done < p.pieces; done++) {
    const int64_t i = p.pieces - 1 - done;  // the kept piece first
    const int64_t v0 = i * p.piece, width = V - v0 < p.piece ? V - v0 : p.piece;
    const Matrix wp{static_cast<const char*>(w.p) + 2 * v0 * w.ld, width, D, w.ld};
    const Matrix pm{probs, T, width, p.piece};
    if (i != kept) {
      const Shape shape{T, width, D};
      iwp_tc::Problems<1> work;
      if (!make_problem(&work.p[0], h, true, wp, true, a->dtype, pick_tile_n(shape, pairs), 1)) return IWP_ERR_CUDA;
      work.status = &hdr->status;
      work.early = 0;
      H::Probs::Args pa{};
      pa.en = en;
      pa.lse = a->lse;
      pa.out = probs;
      pa.T = T;
      pa.ld = p.piece;
      pa.v0 = static_cast<int>(v0);
      pa.width = static_cast<int>(width);
      pa.c = c;
      pa.up = up;
      pa.type = a->dtype;
      if (!make_map(&pa.map, probs, T, p.piece, p.piece, 32, a->dtype)) return IWP_ERR_CUDA;
      if (int e = launch_product<H::Probs, 1>(work, pa, pairs, st)) return e;
    }
    // both gradients of the piece in one launch, dhidden (the longer tiles) first
    iwp_tc::Problems<2> work;
    work.p[0].m_tiles = work.p[0].n_tiles = work.p[0].splits = 0;
    work.p[1].m_tiles = work.p[1].n_tiles = work.p[1].splits = 0;
    work.p[1].use_other = nullptr;
    work.status = &hdr->status;
    work.early = 0;
    const Shape dh{T, D, width}, dw{width, D, T};
    const Deal deal = deal_gradients(a->dhidden ? &dh : nullptr, a->dweight ? &dw : nullptr, pairs, done == 0 ? 0 : splits);
    work.rounds = deal.rounds;
    work.rest = deal.rest;
    work.fill = deal.fill;
    splits = deal.splits;
    const int tile_n = deal.tile_n;
    if (a->dhidden) {
      const bool direct = p.pieces == 1 && splits == 1;
      H::OutMatrix& o = oa.m[0];
      o.rows = static_cast<int>(T);
      o.cols = static_cast<int>(D);
      if (direct) {
        const int size = a->dhidden_type == IWP_F32 ? 4 : 2;
        o.out = a->dhidden;
        o.ld = a->dhidden_ld;
        o.type = a->dhidden_type;
        o.wide = aligned(o.out, 16) && o.ld * size % 16 == 0;
        o.add = a->accumulate;
        if (!copy_map(o)) return IWP_ERR_CUDA;
      } else {
        o.out = ws + p.join;
        o.by_copy = 0;
        o.ld = up_to(D, 4);
        o.split_stride = T * o.ld;
        o.type = IWP_F32;
        o.wide = 1;
        o.add = done > 0;
        o.raw = 1;
      }
      if (!make_problem(&work.p[0], pm, true, wp, false, a->dtype, tile_n, splits)) return IWP_ERR_CUDA;
    }
    if (a->dweight) {
      H::OutMatrix& o = oa.m[1];
      const int size = a->dweight_type == IWP_F32 ? 4 : 2;
      o.out = static_cast<char*>(a->dweight) + size * v0 * a->dweight_ld;
      o.ld = a->dweight_ld;
      o.rows = static_cast<int>(width);
      o.cols = static_cast<int>(D);
      o.type = a->dweight_type;
      o.wide = aligned(o.out, 16) && o.ld * size % 16 == 0;
      o.add = a->accumulate;
      if (!copy_map(o)) return IWP_ERR_CUDA;
      if (!make_problem(&work.p[1], pm, false, h_dw, false, a->dtype, tile_n, 1)) return IWP_ERR_CUDA;
      if (may_clean) {
        if (!make_map(&work.p[1].b_other, h_copy.p, T, D, p.d_pad, iwp_tc::BLOCK_K, a->dtype)) return IWP_ERR_CUDA;
        work.p[1].use_other = &hdr->clean;
      }
    }
    const bool sums = segments(work.p[0]) > 1 || segments(work.p[1]) > 1;
    if (int e = sums ? launch_product<H::Out<true>, 2>(work, oa, pairs, st) : launch_product<H::Out<false>, 2>(work, oa, pairs, st)) return e;
  }
  if (a->dhidden && (p.pieces > 1 || splits > 1)) {
    const int size = a->dhidden_type == IWP_F32 ? 4 : 2;
    const int wide = aligned(a->dhidden, 16) && a->dhidden_ld * size % 16 == 0;
    LOSS_CUDA(launch(H::k_join, T < 16 * sms ? T : 16 * sms, 256, 0, 1, st, oa.f, row_power, reinterpret_cast<const float*>(ws + p.join), splits, T,
                     static_cast<int>(D), a->dhidden, a->dhidden_ld, a->dhidden_type, a->accumulate, wide));
  }
  return IWP_OK;
}

// ---- balance loss -----------------------------------------------------------------------------------------

bool balance_args_ok(const iwp_balance_args* a) {
  if (!a || a->tokens < 0 || a->tokens > MAX_SIZE || a->experts < 1 || a->experts > iwp_balance::MAX_EXPERTS) return false;
  if (a->top_k < 1 || a->top_k > a->experts) return false;
  return a->type == IWP_F32 || a->type == IWP_BF16 || a->type == IWP_F16;
}

constexpr int BALANCE_BLOCKS = 148;  // at most, of the rows kernel
// Up to this many bytes of logits and ids one cluster serves: it saves the second launch and its 16 SMs keep up
// (0.7 MB: 12.6 us in one launch, 19.8 in two; 2.5 MB: 17.1 and 17.8; 5 MB: 25.8 and 15.4).
constexpr int64_t CLUSTER_BYTES = int64_t(3) << 20;

int64_t balance_part_counts_bytes(int E) { return up_to(int64_t(iwp_balance::COUNT_PARTS) * (E + 1) * 4, 256); }

// 16 CTAs (above the portable size, which the kernel has opted in to) where the device can hold such a cluster, else 8.
template <class Kernel>
int largest_cluster(Kernel kernel, int threads, int smem) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(iwp_balance::MAX_CLUSTER);
  cfg.blockDim = dim3(static_cast<unsigned>(threads));
  cfg.dynamicSmemBytes = static_cast<size_t>(smem);
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = iwp_balance::MAX_CLUSTER;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) cudaGetLastError();
  return n > 0 ? iwp_balance::MAX_CLUSTER : 8;
}

template <int TYPE, int VEC, int N>
int balance_launch(iwp_balance::Args a, int G, cudaStream_t st) {
  namespace B = iwp_balance;
  constexpr int threads = B::threads_of(VEC * N), slots = B::slot_bytes(VEC * N, TYPE == IWP_F32 ? 4 : 2);
  auto kernel = B::k_balance_rows<TYPE, VEC, N>;
  static std::atomic<bool> ready[MAX_DEVICES] = {};
  static std::atomic<int> cluster[MAX_DEVICES] = {};
  const int dev = device();
  if (dev < 0) return IWP_ERR_CUDA;
  if (!ready[dev]) {
    LOSS_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, slots));
    LOSS_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    cluster[dev] = largest_cluster(kernel, threads, slots);
    ready[dev] = true;
  }
  const int64_t steps = tiles_of(a.T, threads / G);
  const int64_t bytes = a.T * (a.E * (TYPE == IWP_F32 ? 4 : 2) + a.k * a.ids_bytes);
  if (bytes <= CLUSTER_BYTES) {
    // CTAs for about two rounds of rows each
    int ctas = 1;
    while (ctas < cluster[dev] && 2 * ctas < steps) ctas *= 2;
    a.part_counts = nullptr;
    LOSS_CUDA(launch(kernel, ctas, threads, slots, ctas, st, a, G));
    return IWP_OK;
  }
  LOSS_CUDA(launch(B::k_balance_counts, B::COUNT_BLOCKS, B::COUNT_THREADS, 0, B::COUNT_CLUSTER, st, a));
  LOSS_CUDA(launch(kernel, steps < BALANCE_BLOCKS ? steps : BALANCE_BLOCKS, threads, slots, 1, st, a, G));
  return IWP_OK;
}

// A lane holds VEC neighbouring columns at a time (as many as rows are aligned for, up to 16 bytes), N times: 16
// columns, so that few lanes share a row and the sums over a row take few shuffles; fewer or more of them where a
// row has at most 8 columns or more than 512.
template <int TYPE, int VEC>
int balance_rows(const iwp_balance::Args& a, cudaStream_t st) {
  constexpr int LITTLE = VEC >= 8 ? 8 : 4, LARGE = iwp_balance::MAX_EXPERTS / 32;
  const int columns = a.E <= 8 ? LITTLE : a.E <= 512 ? 16 : LARGE;
  int G = 1;
  while (G * columns < a.E) G *= 2;
  if (columns == LITTLE) return balance_launch<TYPE, VEC, LITTLE / VEC>(a, G, st);
  if (columns == 16) return balance_launch<TYPE, VEC, 16 / VEC>(a, G, st);
  return balance_launch<TYPE, VEC, LARGE / VEC>(a, G, st);
}

template <int TYPE>
int balance_type(const iwp_balance::Args& a, cudaStream_t st) {
  constexpr int size = TYPE == IWP_F32 ? 4 : 2;
  auto fits = [&](int vec) {
    return a.E % vec == 0 && a.logits_ld % vec == 0 && a.dlogits_ld % vec == 0 && aligned(a.logits, vec * size) && aligned(a.dlogits, vec * size);
  };
  if constexpr (size == 2)
    if (fits(8)) return balance_rows<TYPE, 8>(a, st);
  if (fits(4)) return balance_rows<TYPE, 4>(a, st);
  if (fits(2)) return balance_rows<TYPE, 2>(a, st);
  return balance_rows<TYPE, 1>(a, st);
}

}  // namespace

extern "C" int iwp_loss_reset(void* state, void* cuda_stream) {
  if (!state) return IWP_ERR_INVALID;
  LOSS_CUDA(cudaMemsetAsync(state, 0, IWP_LOSS_STATE, static_cast<cudaStream_t>(cuda_stream)));
  return IWP_OK;
}

extern "C" int iwp_loss_status(const void* state, int32_t* status_host, void* cuda_stream) {
  if (!state || !status_host) return IWP_ERR_INVALID;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  LOSS_CUDA(cudaMemcpyAsync(status_host, state, sizeof(int32_t), cudaMemcpyDeviceToHost, st));
  LOSS_CUDA(cudaStreamSynchronize(st));
  return IWP_OK;
}

#ifdef IWP_DEBUG_CHECKS
// Checked build only: a kernel whose bounded waits run out.  gave_up: int, on the device.
extern "C" int iwp_loss_wait_probe(void* state, int32_t* gave_up, void* cuda_stream) {
  if (!state || !gave_up) return IWP_ERR_INVALID;
  LOSS_CUDA(launch(iwp_tc::k_wait_probe, 1, 64, 0, 1, static_cast<cudaStream_t>(cuda_stream), static_cast<int*>(state), gave_up));
  return IWP_OK;
}
#endif

extern "C" int64_t iwp_head_workspace(const iwp_head_args* a) {
  if (!head_args_ok(a)) return -1;
  return head_plan(a).bytes;
}

extern "C" int iwp_head_loss(const iwp_head_args* a, void* cuda_stream) {
  if (!head_args_ok(a)) return IWP_ERR_INVALID;
  if (!a->hidden || !a->weight || !a->lse || !a->workspace || !aligned(a->workspace, 256) || !aligned(a->state, 256)) return IWP_ERR_INVALID;
  if (!aligned(a->hidden, 2) || !aligned(a->weight, 2)) return IWP_ERR_INVALID;
  if (a->dhidden && !aligned(a->dhidden, a->dhidden_type == IWP_F32 ? 4 : 2)) return IWP_ERR_INVALID;
  if (a->dweight && !aligned(a->dweight, a->dweight_type == IWP_F32 ? 4 : 2)) return IWP_ERR_INVALID;
  if (!std::isfinite(a->scale)) return IWP_ERR_INVALID;
  for (const void* x : {static_cast<const void*>(a->loss), static_cast<const void*>(a->rows), static_cast<const void*>(a->lse),
                        static_cast<const void*>(a->dloss), static_cast<const void*>(a->dloss_rows)})
    if (!aligned(x, 4)) return IWP_ERR_INVALID;
  if (!aligned(a->targets, 8)) return IWP_ERR_INVALID;
  if (!a->targets) {
    if (!aligned(a->top_ids, a->ids_bytes == 8 ? 8 : 4) || !aligned(a->top_logits, a->top_type == IWP_F32 ? 4 : 2)) return IWP_ERR_INVALID;
    if (!a->top_ids || !a->top_logits || a->top_ids_ld < a->top_k || a->top_logits_ld < a->top_k) return IWP_ERR_INVALID;
    if ((a->ids_bytes != 4 && a->ids_bytes != 8) || a->top_type < IWP_F32 || a->top_type > IWP_F16) return IWP_ERR_INVALID;
    if (!(a->temperature > 0.f) || !std::isfinite(a->temperature)) return IWP_ERR_INVALID;
  }
  const HeadPlan p = head_plan(a);
  if (a->have_lse && !p.grad) return IWP_ERR_INVALID;
  if (a->workspace_bytes < p.bytes) return IWP_ERR_CAPACITY;
  return head_run(a, p, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" int64_t iwp_balance_workspace(const iwp_balance_args* a) {
  if (!balance_args_ok(a)) return -1;
  return IWP_LOSS_STATE + balance_part_counts_bytes(a->experts) + up_to(int64_t(BALANCE_BLOCKS) * iwp_balance::padded(a->experts) * 4, 256);
}

extern "C" int iwp_balance_loss(const iwp_balance_args* a, void* cuda_stream) {
  if (!balance_args_ok(a)) return IWP_ERR_INVALID;
  const int size = a->type == IWP_F32 ? 4 : 2;
  if (!a->logits || !a->ids || !a->counts || !a->workspace || !aligned(a->workspace, 256) || !aligned(a->state, 256)) return IWP_ERR_INVALID;
  if (a->logits_ld < a->experts || a->ids_ld < a->top_k || (a->ids_bytes != 4 && a->ids_bytes != 8)) return IWP_ERR_INVALID;
  if (a->dlogits && a->dlogits_ld < a->experts) return IWP_ERR_INVALID;
  if (!aligned(a->logits, size) || (a->dlogits && !aligned(a->dlogits, size)) || !aligned(a->ids, a->ids_bytes)) return IWP_ERR_INVALID;
  if (!aligned(a->loss, 4) || !aligned(a->counts, 4) || !aligned(a->mean_prob, 4) || !aligned(a->dloss, 4)) return IWP_ERR_INVALID;
  if (a->tokens * a->experts > MAX_ELEMENTS || a->logits_ld > MAX_SIZE || a->dlogits_ld > MAX_SIZE || a->ids_ld > MAX_SIZE) return IWP_ERR_INVALID;
  if (!std::isfinite(a->coef) || !std::isfinite(a->scale)) return IWP_ERR_INVALID;
  if (a->workspace_bytes < iwp_balance_workspace(a)) return IWP_ERR_CAPACITY;
  char* const ws = static_cast<char*>(a->workspace);
  iwp_balance::Args r{};
  r.hdr = static_cast<iwp_balance::Header*>(a->state ? a->state : a->workspace);
  r.counts = a->counts;
  r.logits = a->logits;
  r.ids = a->ids;
  r.mask = a->mask;
  r.dloss = a->dloss;
  r.dlogits = a->dlogits;
  r.part_counts = reinterpret_cast<int*>(ws + IWP_LOSS_STATE);
  r.part = reinterpret_cast<float*>(ws + IWP_LOSS_STATE + balance_part_counts_bytes(a->experts));
  r.loss = a->loss;
  r.mean_prob = a->mean_prob;
  r.logits_ld = a->logits_ld;
  r.dlogits_ld = a->dlogits ? a->dlogits_ld : a->logits_ld;
  r.ids_ld = a->ids_ld;
  r.T = a->tokens;
  r.E = a->experts;
  r.k = a->top_k;
  r.ids_bytes = a->ids_bytes;
  r.coef = a->coef;
  r.scale = a->scale;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (a->type == IWP_F32) return balance_type<IWP_F32>(r, st);
  if (a->type == IWP_BF16) return balance_type<IWP_BF16>(r, st);
  return balance_type<IWP_F16>(r, st);
}
