"""Two threads whose first calls of one kernel need different amounts of shared memory: host code alone, the CUDA runtime's calls
are stood in for."""
import os
import subprocess

from paper_1901_01544_b200 import build

SOURCE = r"""
#include <cuda_runtime.h>

#include <cstdio>
#include <map>
#include <thread>

static std::map<const void*, int> limit;
static std::thread other;
static void (*at_first)() = nullptr;
template <class Kernel>
cudaError_t fake_set(Kernel kernel, cudaFuncAttribute, int bytes) {
  limit[reinterpret_cast<const void*>(kernel)] = bytes;
  if (auto* f = at_first) {  // another thread's whole call falls between this one's opting in and its noting it down
    at_first = nullptr;
    other = std::thread(f);
    other.join();
  }
  return cudaSuccess;
}
template <class Kernel, class... Args>
cudaError_t fake_launch(const cudaLaunchConfig_t* cfg, Kernel kernel, Args&&...) {
  const auto it = limit.find(reinterpret_cast<const void*>(kernel));
  const size_t most = it == limit.end() ? 48 * 1024 : it->second;
  return cfg->dynamicSmemBytes <= most ? cudaSuccess : cudaErrorInvalidValue;
}
static cudaError_t fake_device(int* dev) { return *dev = 0, cudaSuccess; }
static cudaError_t fake_last() { return cudaSuccess; }
#define cudaFuncSetAttribute fake_set
#define cudaLaunchKernelEx fake_launch
#define cudaGetDevice fake_device
#define cudaGetLastError fake_last
#define IWP_ROUTE_TYPE IWP_F32
#include "iwp_route_launch.hpp"

static int call(int groups) {
  iwp_router::Args a{};
  a.T = 64, a.E = 256, a.k = 4, a.groups = groups, a.top_groups = 1, a.group_top = 1;
  return iwp_router::launch_route_form<IWP_F32, 32, 8, true>(a, 4, nullptr);
}
int main() {
  using namespace iwp_router;
  if (shared_of(256, 2, 8, 32).bytes <= 48 * 1024 || shared_of(256, 32, 8, 32).bytes <= shared_of(256, 2, 8, 32).bytes) return 3;
  at_first = [] { call(2); };
  const int first = call(32), small = call(2), large = call(32);
  // no call of a kernel needs more than what it opts in to
  int beyond = 0;
  for (int groups = 1; groups <= MAX_GROUPS; groups++) beyond += call(groups) != IWP_OK;
  std::printf("%d %d %d %d\n", first, small, large, beyond);
  return first || small || large || beyond;
}
"""


def test_calls_on_two_threads_leave_room_for_the_larger(tmp_path):
    src = tmp_path / "t.cu"
    src.write_text(SOURCE)
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.run([nvcc, *build.NVCC_FLAGS, "-O1", "-I", build.CSRC, str(src), "-o", str(tmp_path / "t")], check=True, capture_output=True)
    r = subprocess.run([str(tmp_path / "t")], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
