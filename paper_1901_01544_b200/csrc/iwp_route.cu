// iwp_route.cu - C entries of the router and of the exchange (include/iwp_route.h): argument checks and launches.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "iwp_exchange.cuh"
#include "iwp_host.hpp"
#include "iwp_route_launch.hpp"

namespace {

using namespace iwp_host;

constexpr int64_t MAX_SIZE = 0x7FFFFFFF - 0xFFFF;  // of tokens, pairs, widths and strides
constexpr int64_t MAX_ELEMENTS = int64_t(1) << 46;
constexpr int64_t MAX_PAIRS = int64_t(1) << 30;  // room for the steps behind the last one

int size_of(int type) { return type == IWP_F32 ? 4 : 2; }
bool is_type(int type) { return type == IWP_F32 || type == IWP_BF16 || type == IWP_F16; }

// Calls f(type, elements of a word): words of up to 16 bytes that `fits`.
template <int TYPE, class Fits, class F>
int by_word(const Fits& fits, const F& f) {
  using Type = std::integral_constant<int, TYPE>;
  if constexpr (TYPE != IWP_F32)
    if (fits(8)) return f(Type{}, std::integral_constant<int, 8>{});
  if (fits(4)) return f(Type{}, std::integral_constant<int, 4>{});
  if (fits(2)) return f(Type{}, std::integral_constant<int, 2>{});
  return f(Type{}, std::integral_constant<int, 1>{});
}
template <class Fits, class F>
int by_type_and_word(int type, const Fits& fits, const F& f) {
  if (type == IWP_F32) return by_word<IWP_F32>(fits, f);
  if (type == IWP_BF16) return by_word<IWP_BF16>(fits, f);
  return by_word<IWP_F16>(fits, f);
}

// ---- routing ------------------------------------------------------------------------------------------

// Elements of the widest word of up to 16 bytes that rows fit.
template <class Fits>
int widest_word(int type, const Fits& fits) {
  for (int vec = 16 / size_of(type); vec > 1; vec /= 2)
    if (fits(vec)) return vec;
  return 1;
}

bool route_sizes_ok(int64_t T, int E, int k) {
  return T >= 0 && T <= MAX_PAIRS && E >= 1 && E <= iwp_router::MAX_EXPERTS && k >= 1 && k <= iwp_router::MAX_TOP && k <= E && T * E <= MAX_ELEMENTS;
}

// ---- exchange -----------------------------------------------------------------------------------------

bool order_args_ok(const iwp_order_args* a) {
  return a && a->tokens >= 0 && a->experts >= 1 && a->experts <= iwp_exchange::MAX_EXPERTS && a->top_k >= 1 && a->top_k <= iwp_exchange::MAX_TOP &&
         a->tokens <= MAX_PAIRS / a->top_k;
}

// Up to this many pairs one block serves, in one launch, which takes the host 2.5 us less.  (One launch and two, in a loop of calls and
// in a graph: 4096 pairs of 128 experts 11.6 and 14.0, 8.3 and 7.4 us; 6144 pairs 11.8 and 14.1, 11.5 and 7.6; 8192 pairs 14.4 and 14.2, 14.0 and
// 7.6; 16384 pairs 24.3 and 13.2, 23.9 and 7.7.)
constexpr int64_t ONE_BLOCK_PAIRS = 8192;
constexpr int64_t PAIRS_PER_BLOCK = 2048, MAX_ORDER_BLOCKS = 128;

int64_t order_blocks(int64_t pairs) { return pairs <= ONE_BLOCK_PAIRS ? 1 : std::min(MAX_ORDER_BLOCKS, tiles_of(pairs, PAIRS_PER_BLOCK)); }

enum { DISPATCH, COMBINE, COMBINE_GRAD };

bool matrix_ok(const void* p, int64_t ld, int64_t dim, int size) { return p && aligned(p, size) && ld >= dim && ld <= MAX_SIZE; }

int exchange(const iwp_exchange_args* a, int what, cudaStream_t st) {
  namespace X = iwp_exchange;
  if (!a || a->tokens < 0 || a->top_k < 1 || a->top_k > X::MAX_TOP || a->experts < 1 || a->experts > X::MAX_EXPERTS) return IWP_ERR_INVALID;
  if (a->tokens > MAX_PAIRS / a->top_k || a->dim < 1 || a->dim > MAX_SIZE || !is_type(a->type)) return IWP_ERR_INVALID;
  if (a->tokens * a->top_k * a->dim > MAX_ELEMENTS) return IWP_ERR_INVALID;
  const int size = size_of(a->type);
  if (!a->slots || !a->offsets || !aligned(a->slots, 4) || !aligned(a->offsets, 4)) return IWP_ERR_INVALID;
  const bool reads_token = what != COMBINE, reads_slot = what == COMBINE || (what == COMBINE_GRAD && a->dweights);
  const bool writes_slot = what == DISPATCH || (what == COMBINE_GRAD && a->by_slot_out);
  if (reads_token && !matrix_ok(a->by_token, a->by_token_ld, a->dim, size)) return IWP_ERR_INVALID;
  if (reads_slot && !matrix_ok(a->by_slot, a->by_slot_ld, a->dim, size)) return IWP_ERR_INVALID;
  if (writes_slot && !matrix_ok(a->by_slot_out, a->by_slot_out_ld, a->dim, size)) return IWP_ERR_INVALID;
  if (what == COMBINE && !matrix_ok(a->by_token_out, a->by_token_out_ld, a->dim, size)) return IWP_ERR_INVALID;
  if (what == COMBINE_GRAD && !a->dweights && !a->by_slot_out) return IWP_ERR_INVALID;
  if (a->weights && (a->weights_ld < a->top_k || a->weights_ld > MAX_SIZE || !aligned(a->weights, 4))) return IWP_ERR_INVALID;
  if (!aligned(a->dweights, 4)) return IWP_ERR_INVALID;
  if (a->tokens == 0) return IWP_OK;
  X::RowArgs r{};
  r.slots = a->slots;
  r.used = a->offsets + a->experts;
  r.by_token = reads_token ? a->by_token : nullptr;
  r.by_slot = reads_slot ? a->by_slot : nullptr;
  r.weights = a->weights;
  r.by_token_out = what == COMBINE ? a->by_token_out : nullptr;
  r.by_slot_out = writes_slot ? a->by_slot_out : nullptr;
  r.dweights = what == COMBINE_GRAD ? a->dweights : nullptr;
  r.by_token_ld = reads_token ? a->by_token_ld : 0;
  r.by_slot_ld = reads_slot ? a->by_slot_ld : 0;
  r.weights_ld = a->weights_ld;
  r.by_token_out_ld = what == COMBINE ? a->by_token_out_ld : 0;
  r.by_slot_out_ld = writes_slot ? a->by_slot_out_ld : 0;
  r.T = static_cast<int>(a->tokens);
  r.D = static_cast<int>(a->dim);
  r.k = a->top_k;
  auto fits = [&](int vec) {
    auto one = [&](const void* p, int64_t ld) { return !p || (aligned(p, vec * size) && (ld % vec == 0 || a->tokens * a->top_k == 1)); };
    return a->dim % vec == 0 && one(r.by_token, r.by_token_ld) && one(r.by_slot, r.by_slot_ld) && one(r.by_token_out, r.by_token_out_ld) &&
           one(r.by_slot_out, r.by_slot_out_ld);
  };
  return by_type_and_word(a->type, fits, [&](auto type, auto vec) -> int {
    constexpr int TYPE = decltype(type)::value, VEC = decltype(vec)::value;
    const int64_t words = a->dim / VEC;
    X::RowArgs q = r;
    if (what == COMBINE_GRAD) {
      const int threads = static_cast<int>(std::min<int64_t>(X::ROW_THREADS, up_to(words, 32)));
      const int64_t blocks = std::min<int64_t>(a->tokens, int64_t(16) * SMS * X::ROW_THREADS / threads);
      if (a->top_k <= 8)
        LOSS_CUDA(launch(X::k_combine_grad<TYPE, VEC, 8>, blocks, threads, 0, 1, st, q));
      else
        LOSS_CUDA(launch(X::k_combine_grad<TYPE, VEC, 32>, blocks, threads, 0, 1, st, q));
      return IWP_OK;
    }
    if (what == COMBINE) {
      const int threads = static_cast<int>(std::min<int64_t>(X::ROW_THREADS, up_to(words, 32)));
      q.parts = static_cast<int>(tiles_of(words, threads));
      const int64_t blocks = std::min<int64_t>(a->tokens * q.parts, int64_t(6) * SMS * X::ROW_THREADS / threads);
      LOSS_CUDA(launch(X::k_combine<TYPE, VEC>, blocks, threads, 0, 1, st, q));
      return IWP_OK;
    }
    // few tokens: several warps share a row, down to a word per lane
    q.parts = 1;
    while (a->tokens * q.parts < int64_t(8) * SMS * X::ROW_WARPS && words / (2 * q.parts) >= 32) q.parts *= 2;
    const int64_t blocks = std::min<int64_t>(tiles_of(a->tokens * q.parts, X::ROW_WARPS), int64_t(8) * SMS);
    LOSS_CUDA(launch(X::k_dispatch<TYPE, VEC>, blocks, X::ROW_THREADS, 0, 1, st, q));
    return IWP_OK;
  });
}

}  // namespace

extern "C" int iwp_route_reset(void* state, void* cuda_stream) {
  if (!state) return IWP_ERR_INVALID;
  LOSS_CUDA(cudaMemsetAsync(state, 0, IWP_ROUTE_STATE, static_cast<cudaStream_t>(cuda_stream)));
  return IWP_OK;
}

extern "C" int iwp_route(const iwp_route_args* a, void* cuda_stream) {
  if (!a || !route_sizes_ok(a->tokens, a->experts, a->top_k) || !is_type(a->type)) return IWP_ERR_INVALID;
  if (a->groups < 1 || a->groups > iwp_router::MAX_GROUPS || a->experts % a->groups || a->top_groups < 1 || a->top_groups > a->groups) return IWP_ERR_INVALID;
  if (a->group_top < 1 || a->group_top > 2 || (a->groups > 1 && a->group_top > a->experts / a->groups)) return IWP_ERR_INVALID;
  if (a->top_k > a->experts / a->groups * a->top_groups) return IWP_ERR_INVALID;
  if (a->score != IWP_SOFTMAX && a->score != IWP_SIGMOID) return IWP_ERR_INVALID;
  if (!std::isfinite(a->weight_scale) || a->weight_scale == 0.f || (a->ids_bytes != 4 && a->ids_bytes != 8)) return IWP_ERR_INVALID;
  if (!a->logits || !a->ids || !a->weights || !a->state || !aligned(a->state, 256)) return IWP_ERR_INVALID;
  const int size = size_of(a->type);
  if (a->logits_ld < a->experts || a->logits_ld > MAX_SIZE || !aligned(a->logits, size) || !aligned(a->ids, a->ids_bytes)) return IWP_ERR_INVALID;
  if (!aligned(a->weights, 4) || !aligned(a->bias, 4) || !aligned(a->counts, 4)) return IWP_ERR_INVALID;
  iwp_router::Args r{};
  r.state = static_cast<iwp_router::State*>(a->state);
  r.logits = a->logits;
  r.bias = a->bias;
  r.mask = a->mask;
  r.ids = a->ids;
  r.weights = a->weights;
  r.counts = a->counts;
  r.logits_ld = a->logits_ld;
  r.T = static_cast<int>(a->tokens);
  r.weight_scale = a->weight_scale;
  r.E = a->experts;
  r.k = a->top_k;
  r.groups = a->top_groups == a->groups ? 1 : a->groups;  // all groups take part: no choice among them
  r.top_groups = a->top_groups;
  r.group_top = a->group_top;
  r.score = a->score;
  r.renormalize = a->renormalize != 0;
  r.ids_bytes = a->ids_bytes;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  auto fits = [&](int vec) { return a->experts % vec == 0 && (a->logits_ld % vec == 0 || a->tokens == 1) && aligned(a->logits, vec * size); };
  const int word = widest_word(a->type, fits);
  if (a->type == IWP_F32) return iwp_router::launch_route<IWP_F32>(r, word, st);
  if (a->type == IWP_BF16) return iwp_router::launch_route<IWP_BF16>(r, word, st);
  return iwp_router::launch_route<IWP_F16>(r, word, st);
}

extern "C" int iwp_route_grad(const iwp_route_grad_args* a, void* cuda_stream) {
  if (!a || !route_sizes_ok(a->tokens, a->experts, a->top_k) || !is_type(a->type)) return IWP_ERR_INVALID;
  if (a->score != IWP_SOFTMAX && a->score != IWP_SIGMOID) return IWP_ERR_INVALID;
  if (!std::isfinite(a->weight_scale) || a->weight_scale == 0.f || !std::isfinite(a->scale) || (a->ids_bytes != 4 && a->ids_bytes != 8)) return IWP_ERR_INVALID;
  if (!a->logits || !a->ids || !a->weights || !a->dweights || !a->dlogits) return IWP_ERR_INVALID;
  const int size = size_of(a->type);
  if (a->logits_ld < a->experts || a->dlogits_ld < a->experts || a->ids_ld < a->top_k || a->weights_ld < a->top_k || a->dweights_ld < a->top_k) return IWP_ERR_INVALID;
  for (const int64_t ld : {a->logits_ld, a->dlogits_ld, a->ids_ld, a->weights_ld, a->dweights_ld})
    if (ld > MAX_SIZE) return IWP_ERR_INVALID;
  if (!aligned(a->logits, size) || !aligned(a->dlogits, size) || !aligned(a->ids, a->ids_bytes) || !aligned(a->weights, 4) || !aligned(a->dweights, 4))
    return IWP_ERR_INVALID;
  if (a->tokens == 0) return IWP_OK;
  iwp_router::GradArgs r{};
  r.logits = a->logits;
  r.ids = a->ids;
  r.weights = a->weights;
  r.dweights = a->dweights;
  r.dlogits = a->dlogits;
  r.logits_ld = a->logits_ld;
  r.ids_ld = a->ids_ld;
  r.weights_ld = a->weights_ld;
  r.dweights_ld = a->dweights_ld;
  r.dlogits_ld = a->dlogits_ld;
  r.T = static_cast<int>(a->tokens);
  r.inv_scale = 1.f / a->weight_scale;
  r.scale = a->scale;
  r.E = a->experts;
  r.k = a->top_k;
  r.score = a->score;
  r.renormalize = a->renormalize != 0;
  r.ids_bytes = a->ids_bytes;
  r.accumulate = a->accumulate != 0;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  auto fits = [&](int vec) {
    return a->experts % vec == 0 && ((a->logits_ld % vec == 0 && a->dlogits_ld % vec == 0) || a->tokens == 1) && aligned(a->logits, vec * size) &&
           aligned(a->dlogits, vec * size);
  };
  const int word = widest_word(a->type, fits);
  if (a->type == IWP_F32) return iwp_router::launch_route_grad<IWP_F32>(r, word, st);
  if (a->type == IWP_BF16) return iwp_router::launch_route_grad<IWP_BF16>(r, word, st);
  return iwp_router::launch_route_grad<IWP_F16>(r, word, st);
}

extern "C" int64_t iwp_order_workspace(const iwp_order_args* a) {
  if (!order_args_ok(a)) return -1;
  return up_to(std::max<int64_t>(1, 4 * MAX_ORDER_BLOCKS * a->experts), 256);
}

extern "C" int iwp_order(const iwp_order_args* a, void* cuda_stream) {
  namespace X = iwp_exchange;
  if (!order_args_ok(a) || !a->ids || !a->offsets || !a->slots || !a->rows || !a->workspace || !aligned(a->workspace, 256)) return IWP_ERR_INVALID;
  if (a->ids_ld < a->top_k || a->ids_ld > MAX_SIZE || (a->ids_bytes != 4 && a->ids_bytes != 8) || !aligned(a->ids, a->ids_bytes)) return IWP_ERR_INVALID;
  if (!aligned(a->offsets, 4) || !aligned(a->slots, 4) || !aligned(a->rows, 4)) return IWP_ERR_INVALID;
  if (a->workspace_bytes < iwp_order_workspace(a)) return IWP_ERR_CAPACITY;
  const int64_t pairs = a->tokens * a->top_k, blocks = order_blocks(pairs);
  X::OrderArgs r{};
  r.ids = a->ids;
  r.offsets = a->offsets;
  r.slots = a->slots;
  r.rows = a->rows;
  r.part = blocks > 1 ? static_cast<int*>(a->workspace) : nullptr;
  r.ids_ld = a->ids_ld;
  r.pairs = static_cast<int>(pairs);
  r.per_block = static_cast<int>(up_to(tiles_of(pairs, blocks), X::ORDER_THREADS));
  r.E = a->experts;
  r.k = a->top_k;
  r.ids_bytes = a->ids_bytes;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const int smem = 4 * X::ORDER_WARPS * r.E;
  static std::atomic<bool> allowed[MAX_DEVICES] = {};
  LOSS_CUDA(allow_shared(X::k_order_place<4>, 4 * X::ORDER_WARPS * X::MAX_EXPERTS, allowed));
  if (blocks > 1) LOSS_CUDA(launch(X::k_order_count, blocks, X::ORDER_THREADS, 0, 1, st, r));
  LOSS_CUDA(launch(X::k_order_place<4>, blocks, X::ORDER_THREADS, smem, 1, st, r));
  return IWP_OK;
}

extern "C" int iwp_dispatch(const iwp_exchange_args* a, void* cuda_stream) { return exchange(a, DISPATCH, static_cast<cudaStream_t>(cuda_stream)); }
extern "C" int iwp_combine(const iwp_exchange_args* a, void* cuda_stream) { return exchange(a, COMBINE, static_cast<cudaStream_t>(cuda_stream)); }
extern "C" int iwp_combine_grad(const iwp_exchange_args* a, void* cuda_stream) { return exchange(a, COMBINE_GRAD, static_cast<cudaStream_t>(cuda_stream)); }
