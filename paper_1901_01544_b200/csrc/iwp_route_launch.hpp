// iwp_route_launch.hpp - launches of the router's kernels; one translation unit per element type instantiates them.
#pragma once

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "iwp_host.hpp"
#include "iwp_route.cuh"

namespace iwp_router {

// Columns per lane: 8 up to 256 experts, so that a row takes few lanes and what they do together serves several rows.
inline int columns_of(int E) { return E <= 256 ? 8 : E <= 512 ? 16 : 32; }
// Lanes of a row: for its columns, and one for each choice.
inline int lanes_of(int E, int k) {
  int G = 2;
  while (G * columns_of(E) < E || G < k) G *= 2;
  return G;
}

// Calls f(columns per lane, lanes of a row).
template <class F>
int by_layout(int E, int k, const F& f) {
  using C8 = std::integral_constant<int, 8>;
  using L32 = std::integral_constant<int, 32>;
  const int columns = columns_of(E), G = lanes_of(E, k);
  if (columns == 16) return f(std::integral_constant<int, 16>{}, L32{});
  if (columns == 32) return f(L32{}, L32{});
  if (G == 2) return f(C8{}, std::integral_constant<int, 2>{});
  if (G == 4) return f(C8{}, std::integral_constant<int, 4>{});
  if (G == 8) return f(C8{}, std::integral_constant<int, 8>{});
  if (G == 16) return f(C8{}, std::integral_constant<int, 16>{});
  return f(C8{}, L32{});
}

template <int TYPE, int M, int G, bool SCORES>
int launch_route_form(const Args& r, int word, cudaStream_t st) {
  using namespace iwp_host;
  const int smem = shared_of(r.E, r.groups, G, M).bytes;
  const auto kernel = k_route<TYPE, M, G, SCORES>;
  static std::atomic<int> allowed[MAX_DEVICES] = {};
  LOSS_CUDA(allow_shared(kernel, smem, allowed));
  const int64_t steps = tiles_of(r.T, THREADS / G);
  LOSS_CUDA(launch(kernel, std::max<int64_t>(1, std::min<int64_t>(steps, blocks_of(M, SCORES) * SMS)), THREADS, smem, 1, st, r, word));
  return IWP_OK;
}

template <int TYPE>
int launch_route(const Args& r, int word, cudaStream_t st) {
  return by_layout(r.E, r.k, [&](auto columns, auto lanes) {
    constexpr int M = decltype(columns)::value, G = decltype(lanes)::value;
    return r.bias || r.groups > 1 ? launch_route_form<TYPE, M, G, true>(r, word, st) : launch_route_form<TYPE, M, G, false>(r, word, st);
  });
}

template <int TYPE>
int launch_route_grad(const GradArgs& r, int word, cudaStream_t st) {
  return by_layout(r.E, r.k, [&](auto columns, auto lanes) -> int {
    using namespace iwp_host;
    constexpr int M = decltype(columns)::value, G = decltype(lanes)::value;
    const int64_t steps = tiles_of(r.T, THREADS / G);
    LOSS_CUDA(launch(k_route_grad<TYPE, M, G>, std::min<int64_t>(steps, (M == 8 ? 4 : 2) * SMS), THREADS, 0, 1, st, r, word));
    return IWP_OK;
  });
}

#ifndef IWP_ROUTE_TYPE
extern template int launch_route<IWP_F32>(const Args&, int, cudaStream_t);
extern template int launch_route<IWP_BF16>(const Args&, int, cudaStream_t);
extern template int launch_route<IWP_F16>(const Args&, int, cudaStream_t);
extern template int launch_route_grad<IWP_F32>(const GradArgs&, int, cudaStream_t);
extern template int launch_route_grad<IWP_BF16>(const GradArgs&, int, cudaStream_t);
extern template int launch_route_grad<IWP_F16>(const GradArgs&, int, cudaStream_t);
#endif

}  // namespace iwp_router
