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

// The same as bits, in as few registers as they take until a value is needed.
template <int BYTES>
struct RawOf {
  using T = uint4;
};
template <>
struct RawOf<8> {
  using T = uint2;
};
template <>
struct RawOf<4> {
  using T = uint32_t;
};
template <>
struct RawOf<2> {
  using T = uint16_t;
};
template <int TYPE, int VEC>
using Raw = typename RawOf<sizeof(Word<TYPE, VEC>)>::T;

template <int TYPE, int VEC>
__device__ __forceinline__ float element(const Raw<TYPE, VEC>& w, int v) {
  if constexpr (TYPE == IWP_F32) {
    return reinterpret_cast<const float*>(&w)[v];
  } else if constexpr (TYPE == IWP_BF16) {
    if constexpr (VEC == 1) return __uint_as_float(static_cast<uint32_t>(w) << 16);
    const uint32_t two = reinterpret_cast<const uint32_t*>(&w)[v / 2];
    return __uint_as_float(v % 2 ? two & 0xFFFF0000u : two << 16);
  } else {
    if constexpr (VEC == 1) return __half2float(__ushort_as_half(w));
    const float2 two = __half22float2(reinterpret_cast<const __half2*>(&w)[v / 2]);
    return v % 2 ? two.y : two.x;
  }
}

constexpr unsigned ALL = 0xFFFFFFFFu;

// Programmatic launches: a kernel may start while the one before it drains, and touches memory only after the wait.
__device__ __forceinline__ void launch_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

__device__ __forceinline__ int64_t load_id(const void* ids, int bytes, int64_t at) {
  return bytes == 8 ? static_cast<const int64_t*>(ids)[at] : static_cast<const int32_t*>(ids)[at];
}

}  // namespace iwp_elem
