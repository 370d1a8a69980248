// iwp_elem.cuh - what the kernels of the router, the exchange and the clipping share: element types, words, launches.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math_constants.h>

#include <cstdint>

#include "../../include/iwp_loss.h"

namespace iwp_elem {

template <int TYPE>
struct Of {
  using T = float;
};
template <>
struct Of<IWP_BF16> {
  using T = __nv_bfloat16;
};
template <>
struct Of<IWP_F16> {
  using T = __half;
};

// VEC neighbouring elements, moved as one word.
template <int TYPE, int VEC>
struct alignas(sizeof(typename Of<TYPE>::T) * VEC) Word {
  typename Of<TYPE>::T x[VEC];
};

constexpr unsigned ALL = 0xFFFFFFFFu;

// Programmatic launches: a kernel may start while the one before it drains, and touches memory only after the wait.
__device__ __forceinline__ void launch_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

__device__ __forceinline__ int64_t load_id(const void* ids, int bytes, int64_t at) {
  return bytes == 8 ? static_cast<const int64_t*>(ids)[at] : static_cast<const int32_t*>(ids)[at];
}

}  // namespace iwp_elem
