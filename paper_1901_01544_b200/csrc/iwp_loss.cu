// iwp_loss.cu - C entries of the losses (include/iwp_loss.h): argument checks, workspace layout, launches.
#include <cmath>
#include <cstring>

#include "iwp_balance.cuh"
#include "iwp_head.cuh"

namespace {

using iwp_tc::Work;

#define LOSS_CUDA(expr)            \
  do {                             \
    if ((expr) != cudaSuccess) {   \
      cudaGetLastError();          \
      return IWP_ERR_CUDA;         \
    }                              \
  } while (0)

constexpr int64_t MAX_SIZE = 0x7FFFFFFF;
constexpr int64_t DEFAULT_PIECE = int64_t(512) << 20;
constexpr int64_t JOIN_TILES = 2 * 148;  // a split dhidden has at most this many partial tiles

inline int64_t up_to(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
inline int64_t tiles_of(int64_t x, int64_t t) { return (x + t - 1) / t; }
inline bool aligned(const void* p, int64_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

int sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
  return n;
}

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

// A row-major matrix of 16-bit elements, read in boxes of box_rows rows and 64 elements (128 bytes, swizzled).
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

// How many clusters of CG CTAs of this kernel the device holds at once: the persistent grid (a cluster that had to wait
// for another to end would double the time).  Looked up once per device.
template <class Kernel>
int resident_clusters(Kernel kernel, int cg, int smem, int* cached) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
  if (cached[dev]) return cached[dev];
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return 0;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(cg));
  cfg.blockDim = dim3(iwp_tc::THREADS);
  cfg.dynamicSmemBytes = smem;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = cg;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) return 0;
  return cached[dev] = n;
}

struct Matrix {
  const void* p;
  int64_t rows, cols, ld;
};

// C[M, N] = A B^T with M, N, K taken from the operands: a K-contiguous operand is [M or N][K], the other [K][M or N].
template <int CG, bool A_KC, bool B_KC, class Epi>
int launch_product(const Matrix& A, const Matrix& B, int dtype, int splits, const typename Epi::Args& args, int* status,
                   cudaStream_t st) {
  using S = iwp_tc::Shape<CG>;
  CUtensorMap ma, mb;
  if (!make_map(&ma, A.p, A.rows, A.cols, A.ld, A_KC ? iwp_tc::TILE_M : iwp_tc::BLOCK_K, dtype) ||
      !make_map(&mb, B.p, B.rows, B.cols, B.ld, B_KC ? S::B_ROWS : iwp_tc::BLOCK_K, dtype))
    return IWP_ERR_CUDA;
  const int64_t M = A_KC ? A.rows : A.cols, N = B_KC ? B.rows : B.cols, K = A_KC ? A.cols : A.rows;
  Work w;
  w.m_tiles = static_cast<int>(tiles_of(M, iwp_tc::TILE_M * CG));
  w.n_tiles = static_cast<int>(tiles_of(N, iwp_tc::TILE_N));
  w.k_blocks = static_cast<int>(tiles_of(K, iwp_tc::BLOCK_K));
  w.splits = splits;
  // f32 accumulator; operand types; which operands are M/N-contiguous; N / 8; M / 16
  w.idesc = (1u << 4) | ((dtype == IWP_BF16 ? 1u : 0u) << 7) | ((dtype == IWP_BF16 ? 1u : 0u) << 10) | ((A_KC ? 0u : 1u) << 15) |
            ((B_KC ? 0u : 1u) << 16) | ((iwp_tc::TILE_N / 8u) << 17) | ((iwp_tc::TILE_M * CG / 16u) << 24);
  w.status = status;
  const int64_t total = int64_t(w.m_tiles) * w.n_tiles * splits;
  if (total > MAX_SIZE) return IWP_ERR_INVALID;
  auto kernel = iwp_tc::k_product<CG, A_KC, B_KC, Epi>;
  static int resident[64] = {};
  const int clusters = resident_clusters(kernel, CG, S::SMEM, resident);
  if (clusters < 1) {
    cudaGetLastError();
    return IWP_ERR_CUDA;
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(CG * (total < clusters ? total : clusters)));
  cfg.blockDim = dim3(iwp_tc::THREADS);
  cfg.dynamicSmemBytes = S::SMEM;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = CG;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  LOSS_CUDA(cudaLaunchKernelEx(&cfg, kernel, ma, mb, w, args));
  return IWP_OK;
}

// ---- output head ----------------------------------------------------------------------------------------

struct HeadPlan {
  bool grad, pack_hidden, pack_weight;
  int64_t k, parts, piece, p_ld, pieces;
  int splits;
  int64_t d_pad;
  // offsets into the workspace
  int64_t column, q, const_term, row_scale, z_at, block_sum, hidden, weight, big, join, bytes;
};

bool needs_copy(const void* p, int64_t ld) { return !aligned(p, 16) || ld % 8 != 0; }

bool head_args_ok(const iwp_head_args* a) {
  if (!a || a->tokens < 0 || a->tokens > MAX_SIZE || a->vocab < 1 || a->vocab > MAX_SIZE - 1024 || a->dim < 1 || a->dim > MAX_SIZE) return false;
  if (a->dtype != IWP_BF16 && a->dtype != IWP_F16) return false;
  if (!a->targets && (a->top_k < 1 || a->top_k > iwp_head::MAX_TOP)) return false;
  if (a->hidden_ld < a->dim || a->weight_ld < a->dim) return false;
  if (a->dhidden && (a->dhidden_ld < a->dim || (a->dhidden_type != a->dtype && a->dhidden_type != IWP_F32))) return false;
  if (a->dweight && (a->dweight_ld < a->dim || (a->dweight_type != a->dtype && a->dweight_type != IWP_F32))) return false;
  return a->piece_bytes >= 0;
}

HeadPlan head_plan(const iwp_head_args* a) {
  HeadPlan p{};
  const int64_t T = a->tokens, V = a->vocab, D = a->dim;
  p.grad = a->dhidden || a->dweight;
  p.k = a->targets ? 1 : a->top_k;
  p.parts = 2 * tiles_of(V, iwp_tc::TILE_N);
  p.d_pad = up_to(D, 8);
  p.pack_hidden = needs_copy(a->hidden, a->hidden_ld);
  p.pack_weight = needs_copy(a->weight, a->weight_ld);
  int64_t at = 256;
  auto take = [&at](int64_t n) {
    const int64_t o = at;
    at += up_to(n, 256);
    return o;
  };
  p.column = take(4 * p.k * T);
  p.q = take(4 * p.k * T);
  p.const_term = take(4 * T);
  p.row_scale = take(4 * T);
  p.z_at = take(4 * p.k * T);
  p.block_sum = take(4 * tiles_of(T, 32));
  if (p.pack_hidden) p.hidden = take(2 * T * p.d_pad);
  if (p.pack_weight) p.weight = take(2 * V * p.d_pad);
  // one region for the partial statistics of the logits pass and, afterwards, the probabilities of a piece
  int64_t big = a->have_lse ? 0 : 8 * p.parts * T;
  if (p.grad) {
    const int64_t limit = a->piece_bytes ? a->piece_bytes : DEFAULT_PIECE;
    const int64_t v_pad = up_to(V, iwp_tc::TILE_N), t = T > 0 ? T : 1;
    int64_t width = limit / (2 * t) / iwp_tc::TILE_N * iwp_tc::TILE_N;
    if (width < iwp_tc::TILE_N) width = iwp_tc::TILE_N;
    if (width > v_pad) width = v_pad;
    p.pieces = tiles_of(v_pad, width);
    p.piece = up_to(tiles_of(v_pad, p.pieces), iwp_tc::TILE_N);
    p.p_ld = p.piece;
    const int64_t most = 2 * t * v_pad < limit ? 2 * t * v_pad : limit, least = 2 * t * iwp_tc::TILE_N;
    const int64_t bound = most > least ? most : least;
    if (bound > big) big = bound;
    // dhidden: few tiles and a long K are split, so that every SM pair has one; more than one piece is summed in fp32
    const int64_t tiles = tiles_of(t, 2 * iwp_tc::TILE_M) * tiles_of(D, iwp_tc::TILE_N), k_blocks = tiles_of(p.piece, iwp_tc::BLOCK_K);
    int64_t s = 74 / tiles;
    if (s > k_blocks / 8) s = k_blocks / 8;
    p.splits = s < 1 ? 1 : static_cast<int>(s);
  }
  p.big = take(big);
  if (a->dhidden) {
    const int64_t one = 4 * T * D, split = JOIN_TILES * 4 * 2 * iwp_tc::TILE_M * iwp_tc::TILE_N;
    p.join = take(one > split ? one : split);
  }
  p.bytes = at;
  return p;
}

int head_run(const iwp_head_args* a, const HeadPlan& p, cudaStream_t st) {
  namespace H = iwp_head;
  const int64_t T = a->tokens, V = a->vocab, D = a->dim;
  char* const ws = static_cast<char*>(a->workspace);
  auto* hdr = reinterpret_cast<H::Header*>(ws);
  const int sms = sm_count();
  if (sms < 2) return IWP_ERR_CUDA;
  const float tau = a->targets ? 1.f : a->temperature;
  if (T == 0) {
    if (a->loss && !a->have_lse) LOSS_CUDA(cudaMemsetAsync(a->loss, 0, 4, st));
    if (a->dweight && !a->accumulate) {
      const int64_t e = a->dweight_type == IWP_F32 ? 4 : 2;
      LOSS_CUDA(cudaMemset2DAsync(a->dweight, a->dweight_ld * e, 0, D * e, V, st));
    }
    return IWP_OK;
  }
  LOSS_CUDA(cudaMemsetAsync(ws + 4, 0, 12, st));  // counters; the status word stays
  H::Entries en;
  en.column = reinterpret_cast<int*>(ws + p.column);
  en.q = reinterpret_cast<float*>(ws + p.q);
  en.const_term = reinterpret_cast<float*>(ws + p.const_term);
  en.row_scale = reinterpret_cast<float*>(ws + p.row_scale);
  en.k = static_cast<int>(p.k);
  if (a->targets) {
    H::k_hard_targets<<<static_cast<unsigned>(tiles_of(T, 256)), 256, 0, st>>>(hdr, en, a->targets, a->ignore_index, T, V);
  } else {
    H::k_soft_targets<<<static_cast<unsigned>(tiles_of(T, 4)), 128, 4 * 4 * p.k, st>>>(hdr, en, a->top_ids, a->top_ids_ld, a->ids_bytes,
                                                                                   a->top_logits, a->top_logits_ld, a->top_type, 1.f / tau, T, V);
  }
  LOSS_CUDA(cudaGetLastError());
  if (p.grad && a->dloss_rows) {
    H::k_row_scales<<<1, 1024, 0, st>>>(hdr, en.row_scale, a->dloss_rows, T);
    LOSS_CUDA(cudaGetLastError());
  }
  Matrix h{a->hidden, T, D, a->hidden_ld}, w{a->weight, V, D, a->weight_ld};
  if (p.pack_hidden) {
    H::k_align_rows<<<static_cast<unsigned>(T < 8 * sms ? T : 8 * sms), 256, 0, st>>>(static_cast<const uint16_t*>(a->hidden), a->hidden_ld,
                                                                                  reinterpret_cast<uint16_t*>(ws + p.hidden), p.d_pad, T, static_cast<int>(D));
    h.p = ws + p.hidden, h.ld = p.d_pad;
  }
  if (p.pack_weight) {
    H::k_align_rows<<<static_cast<unsigned>(V < 8 * sms ? V : 8 * sms), 256, 0, st>>>(static_cast<const uint16_t*>(a->weight), a->weight_ld,
                                                                                  reinterpret_cast<uint16_t*>(ws + p.weight), p.d_pad, V, static_cast<int>(D));
    w.p = ws + p.weight, w.ld = p.d_pad;
  }
  LOSS_CUDA(cudaGetLastError());
  const float c = H::LOG2E / tau;
  if (!a->have_lse) {
    H::Logits::Args la{};
    la.en = en;
    la.T = T;
    la.V = static_cast<int>(V);
    la.c = c;
    la.part = reinterpret_cast<float2*>(ws + p.big);
    la.z_at = reinterpret_cast<float*>(ws + p.z_at);
    if (int e = launch_product<2, true, true, H::Logits>(h, w, a->dtype, 1, la, &hdr->status, st)) return e;
    H::k_finish<<<static_cast<unsigned>(tiles_of(T, 32)), 1024, 0, st>>>(hdr, en, la.part, static_cast<int>(p.parts), la.z_at, tau, T, a->rows,
                                                                     a->lse, a->loss, a->mean, reinterpret_cast<float*>(ws + p.block_sum));
    LOSS_CUDA(cudaGetLastError());
  }
  if (!p.grad) return IWP_OK;

  H::Factor f{};
  const float up = a->dtype == IWP_F16 ? 8192.f : 1.f;
  f.hdr = hdr;
  f.dloss = a->dloss;
  f.factor = a->scale * tau / up;
  f.mean = a->mean;
  f.by_rows = a->dloss_rows != nullptr;
  for (int64_t i = 0; i < p.pieces; i++) {
    const int64_t v0 = i * p.piece, width = V - v0 < p.piece ? V - v0 : p.piece;
    const Matrix wp{static_cast<const char*>(w.p) + 2 * v0 * w.ld, width, D, w.ld};
    const Matrix probs{ws + p.big, T, width, p.p_ld};
    H::Probs::Args pa{};
    pa.en = en;
    pa.lse = a->lse;
    pa.out = ws + p.big;
    pa.T = T;
    pa.ld = p.p_ld;
    pa.v0 = static_cast<int>(v0);
    pa.width = static_cast<int>(width);
    pa.c = c;
    pa.up = up;
    pa.type = a->dtype;
    if (int e = launch_product<2, true, true, H::Probs>(h, wp, a->dtype, 1, pa, &hdr->status, st)) return e;
    if (a->dweight) {
      H::Out::Args oa{};
      const int size = a->dweight_type == IWP_F32 ? 4 : 2;
      oa.f = f;
      oa.out = static_cast<char*>(a->dweight) + size * v0 * a->dweight_ld;
      oa.ld = a->dweight_ld;
      oa.rows = static_cast<int>(width);
      oa.cols = static_cast<int>(D);
      oa.type = a->dweight_type;
      oa.wide = aligned(oa.out, 16) && a->dweight_ld * size % 16 == 0;
      oa.add = a->accumulate;
      if (int e = launch_product<2, false, false, H::Out>(probs, h, a->dtype, 1, oa, &hdr->status, st)) return e;
    }
    if (a->dhidden) {
      H::Out::Args oa{};
      oa.f = f;
      oa.rows = static_cast<int>(T);
      oa.cols = static_cast<int>(D);
      const bool direct = p.pieces == 1 && p.splits == 1;
      if (direct) {
        const int size = a->dhidden_type == IWP_F32 ? 4 : 2;
        oa.out = a->dhidden;
        oa.ld = a->dhidden_ld;
        oa.type = a->dhidden_type;
        oa.wide = aligned(oa.out, 16) && oa.ld * size % 16 == 0;
        oa.add = a->accumulate;
      } else {
        oa.out = ws + p.join;
        oa.ld = D;
        oa.split_stride = T * D;
        oa.type = IWP_F32;
        oa.wide = D % 4 == 0;
        oa.add = i > 0;
        oa.raw = 1;
      }
      if (int e = launch_product<2, true, false, H::Out>(probs, wp, a->dtype, p.splits, oa, &hdr->status, st)) return e;
    }
  }
  if (a->dhidden && (p.pieces > 1 || p.splits > 1)) {
    const int64_t blocks = tiles_of(T * D, 1024);
    H::k_join<<<static_cast<unsigned>(blocks < 16 * sms ? blocks : 16 * sms), 256, 0, st>>>(
        f, reinterpret_cast<const float*>(ws + p.join), p.splits, T, static_cast<int>(D), a->dhidden, a->dhidden_ld, a->dhidden_type, a->accumulate);
    LOSS_CUDA(cudaGetLastError());
  }
  return IWP_OK;
}

// ---- balance loss -----------------------------------------------------------------------------------------

bool balance_args_ok(const iwp_balance_args* a) {
  if (!a || a->tokens < 0 || a->tokens > MAX_SIZE || a->experts < 1 || a->experts > iwp_balance::MAX_EXPERTS) return false;
  if (a->top_k < 1 || a->top_k > a->experts) return false;
  return a->type == IWP_F32 || a->type == IWP_BF16 || a->type == IWP_F16;
}

constexpr int BALANCE_BLOCKS = 148 * 2;

template <int TYPE, int VEC>
int balance_rows(const iwp_balance::Rows& r, cudaStream_t st) {
  int G = 1;
  while (G < 32 && G * VEC < r.E) G *= 2;
  const int need = static_cast<int>(tiles_of(r.E, int64_t(G) * VEC));
  const int64_t steps = tiles_of(r.T, iwp_balance::ROW_THREADS / G);
  const unsigned grid = static_cast<unsigned>(steps < 1 ? 1 : steps < BALANCE_BLOCKS ? steps : BALANCE_BLOCKS);
  const int B = iwp_balance::ROW_THREADS;
  if (need <= 1)
    iwp_balance::k_balance_rows<TYPE, VEC, 1><<<grid, B, 0, st>>>(r, G);
  else if (need <= 2)
    iwp_balance::k_balance_rows<TYPE, VEC, 2><<<grid, B, 0, st>>>(r, G);
  else if (need <= 4)
    iwp_balance::k_balance_rows<TYPE, VEC, 4><<<grid, B, 0, st>>>(r, G);
  else if (need <= 8)
    iwp_balance::k_balance_rows<TYPE, VEC, 8><<<grid, B, 0, st>>>(r, G);
  else if constexpr (VEC == 1)
    iwp_balance::k_balance_rows<TYPE, VEC, 32><<<grid, B, 0, st>>>(r, G);
  LOSS_CUDA(cudaGetLastError());
  return IWP_OK;
}

}  // namespace

extern "C" int iwp_loss_reset(void* workspace, void* cuda_stream) {
  if (!workspace) return IWP_ERR_INVALID;
  LOSS_CUDA(cudaMemsetAsync(workspace, 0, 256, static_cast<cudaStream_t>(cuda_stream)));
  return IWP_OK;
}

extern "C" int iwp_loss_status(const void* workspace, int32_t* status_host, void* cuda_stream) {
  if (!workspace || !status_host) return IWP_ERR_INVALID;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  LOSS_CUDA(cudaMemcpyAsync(status_host, workspace, sizeof(int32_t), cudaMemcpyDeviceToHost, st));
  LOSS_CUDA(cudaStreamSynchronize(st));
  return IWP_OK;
}

extern "C" int64_t iwp_head_workspace(const iwp_head_args* a) {
  if (!head_args_ok(a)) return -1;
  return head_plan(a).bytes;
}

extern "C" int iwp_head_loss(const iwp_head_args* a, void* cuda_stream) {
  if (!head_args_ok(a)) return IWP_ERR_INVALID;
  if (!a->hidden || !a->weight || !a->lse || !a->workspace || !aligned(a->workspace, 256)) return IWP_ERR_INVALID;
  if (!aligned(a->hidden, 2) || !aligned(a->weight, 2)) return IWP_ERR_INVALID;
  if (a->dhidden && !aligned(a->dhidden, a->dhidden_type == IWP_F32 ? 4 : 2)) return IWP_ERR_INVALID;
  if (a->dweight && !aligned(a->dweight, a->dweight_type == IWP_F32 ? 4 : 2)) return IWP_ERR_INVALID;
  if (!std::isfinite(a->scale)) return IWP_ERR_INVALID;
  if (!a->targets) {
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
  return 256 + up_to(int64_t(BALANCE_BLOCKS) * a->experts * 4, 256);
}

extern "C" int iwp_balance_loss(const iwp_balance_args* a, void* cuda_stream) {
  if (!balance_args_ok(a)) return IWP_ERR_INVALID;
  const int size = a->type == IWP_F32 ? 4 : 2;
  if (!a->logits || !a->ids || !a->counts || !a->workspace || !aligned(a->workspace, 256)) return IWP_ERR_INVALID;
  if (a->logits_ld < a->experts || a->ids_ld < a->top_k || (a->ids_bytes != 4 && a->ids_bytes != 8)) return IWP_ERR_INVALID;
  if (a->dlogits && a->dlogits_ld < a->experts) return IWP_ERR_INVALID;
  if (!aligned(a->logits, size) || (a->dlogits && !aligned(a->dlogits, size)) || !aligned(a->ids, a->ids_bytes)) return IWP_ERR_INVALID;
  if (!std::isfinite(a->coef) || !std::isfinite(a->scale)) return IWP_ERR_INVALID;
  if (a->workspace_bytes < iwp_balance_workspace(a)) return IWP_ERR_CAPACITY;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  auto* hdr = static_cast<iwp_balance::Header*>(a->workspace);
  const int E = a->experts;
  LOSS_CUDA(cudaMemsetAsync(static_cast<char*>(a->workspace) + 4, 0, 12, st));
  LOSS_CUDA(cudaMemsetAsync(a->counts, 0, 4 * E, st));
  const int64_t pairs = a->tokens * a->top_k;
  if (pairs > 0) {
    const int64_t blocks = tiles_of(pairs, 1024);
    iwp_balance::k_balance_counts<<<static_cast<unsigned>(blocks < 148 ? blocks : 148), 512, 0, st>>>(hdr, a->counts, a->ids, a->ids_ld, a->ids_bytes,
                                                                                              a->mask, a->tokens, a->top_k, E);
    LOSS_CUDA(cudaGetLastError());
  }
  iwp_balance::Rows r{};
  r.hdr = hdr;
  r.counts = a->counts;
  r.logits = a->logits;
  r.mask = a->mask;
  r.dloss = a->dloss;
  r.dlogits = a->dlogits;
  r.part = reinterpret_cast<float*>(static_cast<char*>(a->workspace) + 256);
  r.loss = a->loss;
  r.mean_prob = a->mean_prob;
  r.logits_ld = a->logits_ld;
  r.dlogits_ld = a->dlogits ? a->dlogits_ld : a->logits_ld;
  r.T = a->tokens;
  r.E = E;
  r.k = a->top_k;
  r.coef = a->coef;
  r.scale = a->scale;
  // whole 16-byte words where every row starts on one and holds whole ones
  const int vec = 16 / size;
  const bool wide = E % vec == 0 && r.logits_ld % vec == 0 && r.dlogits_ld % vec == 0 && aligned(r.logits, 16) && aligned(r.dlogits, 16);
  if (a->type == IWP_F32) return wide ? balance_rows<IWP_F32, 4>(r, st) : balance_rows<IWP_F32, 1>(r, st);
  if (a->type == IWP_BF16) return wide ? balance_rows<IWP_BF16, 8>(r, st) : balance_rows<IWP_BF16, 1>(r, st);
  return wide ? balance_rows<IWP_F16, 8>(r, st) : balance_rows<IWP_F16, 1>(r, st);
}
