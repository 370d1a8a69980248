// iwp_host.hpp - what the C entries around the step share: error handling, sizes, launches.
#pragma once

#include <cuda_runtime.h>

#include <atomic>
#include <cstddef>
#include <cstdint>
#include <utility>

#include "../../include/iwp.h"

namespace iwp_host {

#define LOSS_CUDA(expr)            \
  do {                             \
    if ((expr) != cudaSuccess) {   \
      cudaGetLastError();          \
      return IWP_ERR_CUDA;         \
    }                              \
  } while (0)

inline int64_t up_to(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
inline int64_t tiles_of(int64_t x, int64_t t) { return (x + t - 1) / t; }
inline bool aligned(const void* p, int64_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

constexpr int MAX_DEVICES = 64;
constexpr int SMS = 148;

inline int device() {
  int dev = -1;
  return cudaGetDevice(&dev) == cudaSuccess && dev < MAX_DEVICES ? dev : -1;
}

// Shared memory above the default limit is opted in to once per kernel and device: `most` is what any of the kernel's calls may
// need, the same in all of them, so that threads whose first calls meet set the same limit.
template <class Kernel>
cudaError_t allow_shared(Kernel kernel, int most, std::atomic<bool>* allowed) {
  const int dev = device();
  if (dev < 0) return cudaErrorInvalidDevice;
  if (most <= 48 * 1024 || allowed[dev]) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
  if (e == cudaSuccess) allowed[dev] = true;
  return e;
}

// Launches with programmatic serialisation: the kernel may start while the one before it drains.
template <class... Params, class... Args>
cudaError_t launch(void (*kernel)(Params...), int64_t grid, int block, size_t smem, int cluster, cudaStream_t st, Args&&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(grid));
  cfg.blockDim = dim3(static_cast<unsigned>(block));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = static_cast<unsigned>(cluster);
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);
}

}  // namespace iwp_host
