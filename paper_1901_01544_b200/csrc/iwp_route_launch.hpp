// iwp_route_launch.hpp - launches of the router's kernels; one translation unit per element type instantiates them.
#pragma once

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "iwp_host.hpp"
#include "iwp_route.cuh"

namespace iwp_router {

// Lanes of a row: one for each choice, and few, so that what they do together serves several rows; columns of a lane: 8, 16
// or 32.  (131072 x 256 fp32, 8 choices, in us: 8 lanes of 32 columns 54, 16 of 16 72, 32 of 8 96; 4096 x 256: 7.5, 7.7, 8.7;
// 64 x 256: 5.5, 5.3, 4.8, behind a call's host time of 11.)  Up to 64 experts a lane of 8 columns is done sooner, as long as
// all rows run at once; half as many lanes of 16 pay from about 25000 rows on.  (60 experts bf16, 4 choices, 8 lanes and 4:
// 5003 rows 5.3 and 5.4, with sigmoid and bias 7.0 and 8.4; 24576 rows 8.9 and 7.9; 131072 rows 33 and 20.)
inline int lanes_of(int64_t T, int E, int k) {
  const int columns = T < 24576 ? 8 : 16;
  int G = E <= 2 * columns ? 2 : E <= 4 * columns ? 4 : 8;
  while (G * 32 < E || G < k) G *= 2;
  return G;
}
inline int columns_of(int E, int G) { return E <= 8 * G ? 8 : E <= 16 * G ? 16 : 32; }

// Calls f(columns per lane, lanes of a row).
template <class F>
int by_layout(int64_t T, int E, int k, const F& f) {
  const int G = lanes_of(T, E, k), columns = columns_of(E, G);
  auto few = [&](auto lanes) -> int {
    if (columns == 8) return f(std::integral_constant<int, 8>{}, lanes);
    return f(std::integral_constant<int, 16>{}, lanes);
  };
  auto with = [&](auto lanes) -> int {
    if (columns <= 16) return few(lanes);
    return f(std::integral_constant<int, 32>{}, lanes);
  };
  if (G == 2) return few(std::integral_constant<int, 2>{});
  if (G == 4) return few(std::integral_constant<int, 4>{});
  if (G == 8) return with(std::integral_constant<int, 8>{});
  if (G == 16) return with(std::integral_constant<int, 16>{});
  return with(std::integral_constant<int, 32>{});
}

template <int TYPE, int M, int G, bool SCORES>
int launch_route_form(const Args& r, int word, cudaStream_t st) {
  using namespace iwp_host;
  const int smem = shared_of(r.E, r.groups, G, M).bytes;
  const int most = shared_of(std::min(MAX_EXPERTS, M * G), SCORES ? MAX_GROUPS : 1, G, M).bytes;
  const auto kernel = k_route<TYPE, M, G, SCORES>;
  static std::atomic<bool> allowed[MAX_DEVICES] = {};
  LOSS_CUDA(allow_shared(kernel, most, allowed));
  const int64_t steps = tiles_of(r.T, THREADS / G);
  LOSS_CUDA(launch(kernel, std::max<int64_t>(1, std::min<int64_t>(steps, blocks_of(M, SCORES) * SMS)), THREADS, smem, 1, st, r, word));
  return IWP_OK;
}

template <int TYPE>
int launch_route(const Args& r, int word, cudaStream_t st) {
  return by_layout(r.T, r.E, r.k, [&](auto columns, auto lanes) {
    constexpr int M = decltype(columns)::value, G = decltype(lanes)::value;
    return r.bias || r.groups > 1 ? launch_route_form<TYPE, M, G, true>(r, word, st) : launch_route_form<TYPE, M, G, false>(r, word, st);
  });
}

template <int TYPE>
int launch_route_grad(const GradArgs& r, int word, cudaStream_t st) {
  return by_layout(r.T, r.E, r.k, [&](auto columns, auto lanes) -> int {
    using namespace iwp_host;
    constexpr int M = decltype(columns)::value, G = decltype(lanes)::value;
    const int64_t steps = tiles_of(r.T, THREADS / G);
    LOSS_CUDA(launch(k_route_grad<TYPE, M, G>, std::min<int64_t>(steps, grad_blocks_of(M) * SMS), THREADS, 0, 1, st, r, word));
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
