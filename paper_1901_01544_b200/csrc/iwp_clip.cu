// iwp_clip.cu - C entries of the gradients' norms and clipping (include/iwp_clip.h): the table of the parts, checks, launches.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>
#include <memory>
#include <new>

#include "iwp_clip.cuh"
#include "iwp_host.hpp"

namespace {

using namespace iwp_host;
namespace K = iwp_clipper;

constexpr int64_t MAX_ELEMENTS = int64_t(1) << 46, MAX_PARTS = int64_t(1) << 26, MAX_LD = int64_t(1) << 46;
constexpr int MAX_GROUPS = 1 << 20;
constexpr int64_t MAX_WARPS = int64_t(4) * SMS * K::WARPS;
constexpr int MAX_CLUSTER = 16;
// A part costs a warp as much time as this many elements more: its description and its first elements are waited for.
constexpr int64_t PART_COST = 1024;
// Up to this cost one cluster serves, in one launch, which takes the host 2 us less.  (One launch and two, fp32 elements in one tensor, in a
// loop of calls and in a graph: 100000 8.2 and 10.3, 6.2 and 5.8 us; 300000 8.6 and 10.3, 8.1 and 5.7; 500000 9.2 and 10.3, 8.9 and 6.0; 600000 9.9
// and 10.4, 9.5 and 6.1; 1.2 million 11.3 and 10.4, 10.8 and 7.0.)
constexpr int64_t SMALL_COST = int64_t(1) << 19;
constexpr int64_t SMALL_WARPS = MAX_CLUSTER * (K::SMALL_THREADS / 32);

// The sums of a single group, and of up to FEW_GROUPS that FEW_WARPS leave (of some 4 million elements), are added up by the last block
// of the squares' launch, about 1 us a group; else by a launch of its own, 2 us on the host.  (Clipping in a loop of calls, the one and the
// other: 25 million elements in 1 group 25.5 and 26 us, in 2 30.4 and 27.6, in 8 35 and 26; 4.2 million in 1 group 11.4 and 12.5, in 2 12.6 and
// 12.6, in 8 16.9 and 12.6; 3.5 million in 2 10.6 and 12.5, in 8 15.6 and 12.5; 2 million in 2 10.5 and 12.7, in 8 12.7 and 12.8, in 12 16.2 and 12.7.)
constexpr int FEW_GROUPS = 8;
constexpr int64_t FEW_WARPS = 2560;
// In that launch up to this many groups have a block each, which thousands of sums need, more a warp each.  (Norms of 25 million elements in a
// graph, blocks and warps: 2 groups one of which has nearly all 23.1 and 28.1 us, 16 groups 21.9 and 22.4, 64 21.4 and 21.9, 161 21.7 and 21.6; of 4
// million in 64 groups 5.6 and 5.7, in 161 6.0 and 5.7, in 500 6.3 and 5.8.)
constexpr int BLOCK_GROUPS = 128;

int size_of(int type) { return type == IWP_F32 ? 4 : 2; }
bool is_type(int type) { return type == IWP_F32 || type == IWP_BF16 || type == IWP_F16; }

// Warps that share the work out: all that the two passes run at once (or that the cluster has), but with something to stream
// for each.
int64_t warps_for(int64_t cost) {
  const int64_t most = cost <= SMALL_COST ? SMALL_WARPS : MAX_WARPS;
  return std::min(most, tiles_of(cost, PART_COST + 512));
}

bool tensor_ok(const iwp_clip_tensor& t, int groups) {
  if (t.rows < 0 || t.cols < 0 || t.group < 0 || t.group >= groups || !is_type(t.in_type)) return false;
  if (t.rows == 0 || t.cols == 0) return true;
  if (t.rows > MAX_ELEMENTS || t.cols > MAX_ELEMENTS / t.rows) return false;
  if (!t.in || !aligned(t.in, size_of(t.in_type)) || (t.rows > 1 && (t.in_ld < 0 || t.in_ld > MAX_LD))) return false;
  if (!t.out) return true;
  return is_type(t.out_type) && aligned(t.out, size_of(t.out_type)) && (t.rows == 1 || (t.out_ld >= t.cols && t.out_ld <= MAX_LD));
}

// Walks over all elements, by group and in a group by tensor, and calls f(warp, part) for every part in that order; a warp's
// parts cost `range` at most.  Returns the number of warps.
template <class F>
int64_t each_part(const iwp_clip_tensor* tensors, const int64_t* order, int64_t n, int64_t range, const F& f) {
  constexpr int64_t MOST = int64_t(1) << 30, LEAST = 64;
  int64_t w = 0, left = range;
  bool used = false;
  for (int64_t o = 0; o < n; o++) {
    iwp_clip_tensor t = tensors[order[o]];
    if (t.rows == 0 || t.cols == 0) continue;
    if (t.rows > 1 && t.in_ld == t.cols && (!t.out || t.out_ld == t.cols)) t.cols *= t.rows, t.rows = 1;
    for (int64_t r = 0, c = 0; r < t.rows;) {
      if (left < PART_COST + LEAST) w++, left = range;
      const int64_t most = std::min(MOST, (left - PART_COST) / LEAST * LEAST);
      int64_t rows = 1, cols = std::min(t.cols - c, most);
      if (c == 0 && most >= t.cols) rows = std::min(t.rows - r, most / t.cols);  // whole rows
      K::Part p{};
      p.in = static_cast<const char*>(t.in) + (r * t.in_ld + c) * size_of(t.in_type);
      p.out = t.out ? static_cast<char*>(t.out) + (r * t.out_ld + c) * size_of(t.out_type) : nullptr;
      p.in_ld = t.in_ld;
      p.out_ld = t.out ? t.out_ld : 0;
      p.rows = static_cast<int>(rows);
      p.cols = static_cast<int>(cols);
      p.group = t.group;
      p.in_type = static_cast<int16_t>(t.in_type);
      p.out_type = static_cast<int16_t>(t.out ? t.out_type : t.in_type);
      f(w, p);
      used = true;
      left -= PART_COST + rows * cols;
      c += cols;
      if (c == t.cols) c = 0, r += rows;
    }
  }
  return w + used;
}

// Tensors by group, in the order they are given in.
std::unique_ptr<int64_t[]> order_of(const iwp_clip_tensor* tensors, int64_t n) {
  std::unique_ptr<int64_t[]> order(new (std::nothrow) int64_t[n + 1]);
  if (!order) return nullptr;
  for (int64_t i = 0; i < n; i++) order[i] = i;
  std::sort(order.get(), order.get() + n, [&](int64_t a, int64_t b) { return tensors[a].group != tensors[b].group ? tensors[a].group < tensors[b].group : a < b; });
  return order;
}

// How the work is shared out: ranges of about the least cost that the warps there are suffice for.
struct Shares {
  int64_t warps, range, parts;
};
Shares shares_of(const iwp_clip_tensor* tensors, const int64_t* order, int64_t n, int64_t total) {
  Shares s{};
  if (total == 0) return s;
  auto walk = [&](int64_t range) {
    s.range = range;
    s.parts = 0;
    return each_part(tensors, order, n, range, [&](int64_t, const K::Part&) { s.parts++; });
  };
  walk(MAX_ELEMENTS);
  s.warps = warps_for(total + PART_COST * s.parts);
  int64_t range = up_to(tiles_of(total + PART_COST * s.parts, s.warps), 64) + PART_COST;
  while (walk(range) > s.warps) range += up_to(range / 64, 64);
  return s;
}

struct Table {
  int64_t parts, spans, bytes;  // offsets
};
Table table_of(int64_t warps, int64_t parts, int64_t groups) {
  Table t;
  t.parts = warps * int64_t(sizeof(K::Start));
  t.spans = t.parts + parts * int64_t(sizeof(K::Part));
  t.bytes = up_to(t.spans + groups * int64_t(sizeof(int2)), 256);
  return t;
}

}  // namespace

extern "C" int iwp_clip_layout(const iwp_clip_tensor* tensors, int64_t n, int32_t groups, iwp_clip_sizes* sizes) {
  if (!sizes || n < 0 || (n && !tensors) || groups < 1 || groups > MAX_GROUPS) return IWP_ERR_INVALID;
  int64_t total = 0, rows = 0;
  for (int64_t i = 0; i < n; i++) {
    if (!tensor_ok(tensors[i], groups)) return IWP_ERR_INVALID;
    total += tensors[i].rows * tensors[i].cols;
    const iwp_clip_tensor& t = tensors[i];
    if (t.rows > 1 && t.cols > 0 && (t.in_ld != t.cols || (t.out && t.out_ld != t.cols))) rows += t.rows;
    if (total > MAX_ELEMENTS || rows > MAX_PARTS / 2) return IWP_ERR_INVALID;
  }
  const auto order = order_of(tensors, n);
  if (!order) return IWP_ERR_OOM;
  const Shares shares = shares_of(tensors, order.get(), n, total);
  if (shares.parts > MAX_PARTS) return IWP_ERR_INVALID;
  sizes->parts = shares.parts;
  sizes->warps = shares.warps;
  sizes->range = shares.range;
  sizes->table_bytes = table_of(shares.warps, shares.parts, groups).bytes;
  sizes->workspace_bytes = up_to(8 * (shares.warps + groups), 256);
  return IWP_OK;
}

extern "C" int iwp_clip_table(const iwp_clip_tensor* tensors, int64_t n, int32_t groups, void* table, int64_t table_bytes) {
  iwp_clip_sizes sizes;
  if (const int e = iwp_clip_layout(tensors, n, groups, &sizes)) return e;
  if (!table || !aligned(table, 8)) return IWP_ERR_INVALID;
  if (table_bytes < sizes.table_bytes) return IWP_ERR_CAPACITY;
  const auto order = order_of(tensors, n);
  if (!order) return IWP_ERR_OOM;
  std::memset(table, 0, sizes.table_bytes);
  const int64_t warps = sizes.warps;
  const Table at = table_of(warps, sizes.parts, groups);
  char* const base = static_cast<char*>(table);
  auto* const spans = reinterpret_cast<int2*>(base + at.spans);
  int64_t last = -1, i = 0;
  each_part(tensors, order.get(), n, sizes.range, [&](int64_t w, const K::Part& p) {
    std::memcpy(base + at.parts + i * int64_t(sizeof p), &p, sizeof p);
    auto* const start = reinterpret_cast<K::Start*>(base) + w;
    i++;
    if (w != last) {
      std::memcpy(&start->part, &p, sizeof p);
      start->next = static_cast<int>(i);
      last = w;
    }
    start->end = static_cast<int>(i);
    int2& span = spans[p.group];
    const int place = static_cast<int>(w) + p.group;
    if (span.y == 0) span.x = place;
    span.y = place + 1;
  });
  // (the last warps may be left without elements)
  for (int64_t w = last + 1; w < warps; w++) reinterpret_cast<K::Start*>(base)[w].end = -1;
  return IWP_OK;
}

extern "C" int iwp_clip(const iwp_clip_args* a, void* cuda_stream) {
  if (!a || a->groups < 1 || a->groups > MAX_GROUPS || a->parts < 0 || a->parts > MAX_PARTS || a->warps < 0 || a->warps > MAX_WARPS) return IWP_ERR_INVALID;
  if (!a->table || !aligned(a->table, 16) || !a->squares || !aligned(a->squares, 8) || !a->norms || !aligned(a->norms, 4)) return IWP_ERR_INVALID;
  if (!aligned(a->factors, 4) || (a->write && !a->factors) || !a->state || !aligned(a->state, 256)) return IWP_ERR_INVALID;
  if (!a->workspace || !aligned(a->workspace, 256)) return IWP_ERR_INVALID;
  if (!(a->max_norm >= 0.) || !std::isfinite(a->scale) || a->scale == 0.) return IWP_ERR_INVALID;
  const int64_t warps = a->warps;
  if (a->workspace_bytes < 8 * (warps + a->groups)) return IWP_ERR_CAPACITY;
  const Table at = table_of(warps, a->parts, a->groups);
  const char* const table = static_cast<const char*>(a->table);
  K::Args r{};
  r.hdr = static_cast<K::Header*>(a->state);
  r.starts = reinterpret_cast<const K::Start*>(table);
  r.parts = reinterpret_cast<const K::Part*>(table + at.parts);
  r.spans = reinterpret_cast<const int2*>(table + at.spans);
  r.sums = static_cast<double*>(a->workspace);
  r.warps = static_cast<int>(warps);
  r.squares = a->squares;
  r.norms = a->norms;
  r.factors = a->factors;
  r.max_norm = a->max_norm;
  r.scale = a->scale;
  r.groups = a->groups;
  r.join = a->groups == 1 || (a->groups <= FEW_GROUPS && warps <= FEW_WARPS);
  r.write = a->write != 0;
  r.have_squares = a->have_squares != 0;
  r.drop = a->drop_nonfinite != 0;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (warps <= SMALL_WARPS && a->groups <= 4096) {
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
    while (ctas < largest[dev] && ctas * (K::SMALL_THREADS / 32) < warps) ctas *= 2;
    LOSS_CUDA(launch(K::k_small, ctas, K::SMALL_THREADS, 0, ctas, st, r));
    return IWP_OK;
  }
  const int64_t blocks = std::max<int64_t>(1, tiles_of(warps, K::WARPS));
  if (!a->have_squares) LOSS_CUDA(launch(K::k_squares, blocks, K::THREADS, 0, 1, st, r));
  if (a->have_squares || !r.join)
    LOSS_CUDA(a->groups <= BLOCK_GROUPS ? launch(K::k_groups<true>, a->groups, K::THREADS, 0, 1, st, r)
                                        : launch(K::k_groups<false>, std::min<int64_t>(tiles_of(a->groups, K::WARPS), 8 * SMS), K::THREADS, 0, 1, st, r));
  if (a->write && warps) LOSS_CUDA(launch(K::k_scale, blocks, K::THREADS, 0, 1, st, r));
  return IWP_OK;
}
