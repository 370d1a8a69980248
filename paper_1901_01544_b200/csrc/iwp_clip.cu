// iwp_clip.cu - C entries of the gradients' norms and clipping (include/iwp_clip.h): the table of the parts, checks, launches.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>

#include "iwp_clip.cuh"
#include "iwp_host.hpp"

namespace {

using namespace iwp_host;
namespace K = iwp_clipper;

constexpr int SMS = 148;
constexpr int64_t MAX_ELEMENTS = int64_t(1) << 46, MAX_PARTS = int64_t(1) << 26, MAX_LD = int64_t(1) << 46;
constexpr int MAX_GROUPS = 1 << 20;
constexpr int MAX_CLUSTER = 16;
// Up to this many elements one cluster serves, in one launch.
constexpr int64_t SMALL_ELEMENTS = int64_t(1) << 18;

int size_of(int type) { return type == IWP_F32 ? 4 : 2; }
bool is_type(int type) { return type == IWP_F32 || type == IWP_BF16 || type == IWP_F16; }

// Elements of a part: enough parts for every warp that the GPU holds at once (or that the cluster has) where that leaves
// something to stream per lane, and not so many that adding up their sums counts.
int64_t part_elements(int64_t total) {
  const int64_t warps = total <= SMALL_ELEMENTS ? MAX_CLUSTER * (K::SMALL_THREADS / 32) : int64_t(SMS) * 64;
  return std::min<int64_t>(16384, std::max<int64_t>(512, up_to(tiles_of(total, warps), 256)));
}

bool tensor_ok(const iwp_clip_tensor& t, int groups) {
  if (t.rows < 0 || t.cols < 0 || t.group < 0 || t.group >= groups || !is_type(t.in_type)) return false;
  if (t.rows == 0 || t.cols == 0) return true;
  if (t.rows > MAX_ELEMENTS || t.cols > MAX_ELEMENTS / t.rows) return false;
  if (!t.in || !aligned(t.in, size_of(t.in_type)) || (t.rows > 1 && (t.in_ld < 0 || t.in_ld > MAX_LD))) return false;
  if (!t.out) return true;
  return is_type(t.out_type) && aligned(t.out, size_of(t.out_type)) && (t.rows == 1 || (t.out_ld >= t.cols && t.out_ld <= MAX_LD));
}

// Calls f(part) for every part of a tensor; counts them if f is a counter.
template <class F>
void each_part(iwp_clip_tensor t, int64_t size, const F& f) {
  if (t.rows == 0 || t.cols == 0) return;
  if (t.rows > 1 && t.in_ld == t.cols && (!t.out || t.out_ld == t.cols)) t.cols *= t.rows, t.rows = 1;
  const int64_t cols = std::min(t.cols, size), rows = std::max<int64_t>(1, t.cols > size ? 1 : size / t.cols);
  for (int64_t r = 0; r < t.rows; r += rows)
    for (int64_t c = 0; c < t.cols; c += cols) {
      K::Part p{};
      p.in = static_cast<const char*>(t.in) + (r * t.in_ld + c) * size_of(t.in_type);
      p.out = t.out ? static_cast<char*>(t.out) + (r * t.out_ld + c) * size_of(t.out_type) : nullptr;
      p.in_ld = t.in_ld;
      p.out_ld = t.out ? t.out_ld : 0;
      p.rows = static_cast<int>(std::min(rows, t.rows - r));
      p.cols = static_cast<int>(std::min(cols, t.cols - c));
      p.group = t.group;
      p.in_type = static_cast<int16_t>(t.in_type);
      p.out_type = static_cast<int16_t>(t.out ? t.out_type : t.in_type);
      f(p);
    }
}

int64_t parts_of(iwp_clip_tensor t, int64_t size) {
  if (t.rows == 0 || t.cols == 0) return 0;
  if (t.rows > 1 && t.in_ld == t.cols && (!t.out || t.out_ld == t.cols)) t.cols *= t.rows, t.rows = 1;
  return t.cols > size ? t.rows * tiles_of(t.cols, size) : tiles_of(t.rows, size / t.cols);
}

int64_t firsts_at(int64_t parts) { return up_to(parts * int64_t(sizeof(K::Part)), 256); }

}  // namespace

extern "C" int iwp_clip_layout(const iwp_clip_tensor* tensors, int64_t n, int32_t groups, iwp_clip_sizes* sizes) {
  if (!sizes || n < 0 || (n && !tensors) || groups < 1 || groups > MAX_GROUPS) return IWP_ERR_INVALID;
  int64_t total = 0, parts = 0;
  for (int64_t i = 0; i < n; i++) {
    if (!tensor_ok(tensors[i], groups)) return IWP_ERR_INVALID;
    total += tensors[i].rows * tensors[i].cols;
    if (total > MAX_ELEMENTS) return IWP_ERR_INVALID;
  }
  const int64_t size = part_elements(total);
  for (int64_t i = 0; i < n; i++) {
    parts += parts_of(tensors[i], size);
    if (parts > MAX_PARTS) return IWP_ERR_INVALID;
  }
  sizes->parts = parts;
  sizes->elements = total;
  sizes->table_bytes = firsts_at(parts) + up_to(4 * (int64_t(groups) + 1), 256);
  sizes->workspace_bytes = up_to(std::max<int64_t>(8 * parts, 8), 256);
  return IWP_OK;
}

extern "C" int iwp_clip_table(const iwp_clip_tensor* tensors, int64_t n, int32_t groups, void* table, int64_t table_bytes) {
  iwp_clip_sizes sizes;
  if (const int e = iwp_clip_layout(tensors, n, groups, &sizes)) return e;
  if (!table || !aligned(table, 8)) return IWP_ERR_INVALID;
  if (table_bytes < sizes.table_bytes) return IWP_ERR_CAPACITY;
  std::memset(table, 0, sizes.table_bytes);
  const int64_t size = part_elements(sizes.elements);
  int* const first = reinterpret_cast<int*>(static_cast<char*>(table) + firsts_at(sizes.parts));
  // by group, and in a group by tensor: first[g] counts up from the group's first part while the parts are laid out
  for (int64_t i = 0; i < n; i++) first[tensors[i].group + 1] += static_cast<int>(parts_of(tensors[i], size));
  for (int g = 0; g < groups; g++) first[g + 1] += first[g];
  for (int64_t i = 0; i < n; i++)
    each_part(tensors[i], size, [&](const K::Part& p) { std::memcpy(static_cast<char*>(table) + int64_t(first[p.group]++) * sizeof p, &p, sizeof p); });
  for (int g = groups; g > 0; g--) first[g] = first[g - 1];  // each is now where the next begins
  first[0] = 0;
  return IWP_OK;
}

extern "C" int iwp_clip(const iwp_clip_args* a, void* cuda_stream) {
  if (!a || a->groups < 1 || a->groups > MAX_GROUPS || a->parts < 0 || a->parts > MAX_PARTS || a->elements < 0 || a->elements > MAX_ELEMENTS) return IWP_ERR_INVALID;
  if (!a->table || !aligned(a->table, 16) || !a->squares || !aligned(a->squares, 8) || !a->norms || !aligned(a->norms, 4)) return IWP_ERR_INVALID;
  if (!aligned(a->factors, 4) || (a->write && !a->factors) || !a->state || !aligned(a->state, 256)) return IWP_ERR_INVALID;
  if (!a->workspace || !aligned(a->workspace, 256)) return IWP_ERR_INVALID;
  if (!(a->max_norm >= 0.) || !std::isfinite(a->scale) || a->scale == 0.) return IWP_ERR_INVALID;
  if (a->workspace_bytes < 8 * a->parts) return IWP_ERR_CAPACITY;
  K::Args r{};
  r.hdr = static_cast<K::Header*>(a->state);
  r.parts = static_cast<const K::Part*>(a->table);
  r.first = reinterpret_cast<const int*>(static_cast<const char*>(a->table) + firsts_at(a->parts));
  r.sums = static_cast<double*>(a->workspace);
  r.squares = a->squares;
  r.norms = a->norms;
  r.factors = a->factors;
  r.count = a->parts;
  r.max_norm = a->max_norm;
  r.scale = a->scale;
  r.groups = a->groups;
  r.write = a->write != 0;
  r.have_squares = a->have_squares != 0;
  r.drop = a->drop_nonfinite != 0;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (a->elements <= SMALL_ELEMENTS && a->parts <= 4096 && a->groups <= 4096) {
    static std::atomic<int> largest[MAX_DEVICES] = {};
    const int dev = device();
    if (dev < 0) return IWP_ERR_CUDA;
    if (!largest[dev]) {  // 16 CTAs (above the portable size) where the device can hold such a cluster, else 8
      LOSS_CUDA(cudaFuncSetAttribute(K::k_small, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
      cudaLaunchConfig_t cfg{};
      cfg.gridDim = dim3(MAX_CLUSTER);
      cfg.blockDim = dim3(K::SMALL_THREADS);
      cudaLaunchAttribute at[1];
      at[0].id = cudaLaunchAttributeClusterDimension;
      at[0].val.clusterDim.x = MAX_CLUSTER;
      at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
      cfg.attrs = at;
      cfg.numAttrs = 1;
      int n = 0;
      if (cudaOccupancyMaxActiveClusters(&n, K::k_small, &cfg) != cudaSuccess) cudaGetLastError();
      largest[dev] = n > 0 ? MAX_CLUSTER : 8;
    }
    int ctas = 1;
    while (ctas < largest[dev] && ctas * (K::SMALL_THREADS / 32) < a->parts) ctas *= 2;
    LOSS_CUDA(launch(K::k_small, ctas, K::SMALL_THREADS, 0, ctas, st, r));
    return IWP_OK;
  }
  const int64_t blocks = std::max<int64_t>(1, tiles_of(a->parts, K::WARPS));
  if (a->have_squares)
    LOSS_CUDA(launch(K::k_factors, std::min<int64_t>(tiles_of(a->groups, K::THREADS), SMS), K::THREADS, 0, 1, st, r));
  else
    LOSS_CUDA(launch(K::k_squares, std::min<int64_t>(blocks, 8 * SMS), K::THREADS, 0, 1, st, r));
  if (a->write && a->parts) LOSS_CUDA(launch(K::k_scale, std::min<int64_t>(blocks, 6 * SMS), K::THREADS, 0, 1, st, r));
  return IWP_OK;
}
