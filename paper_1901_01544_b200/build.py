"""Builds the C-ABI library libiwp.so in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libiwp.so")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
STEP_DEPS = [os.path.join(CSRC, f) for f in ("iwp_api.cu", "iwp_device.cuh", "iwp_stream.cuh", "iwp_sample.cuh", "iwp_select.cuh", "iwp_reduce.cuh",
                                            "iwp_threshold.cuh", "iwp_wire.cuh", "iwp_plan.hpp")] + [os.path.join(INCLUDE, "iwp.h")]
LOSS_DEPS = [os.path.join(CSRC, f) for f in ("iwp_loss.cu", "iwp_tensor.cuh", "iwp_head.cuh", "iwp_balance.cuh", "iwp_host.hpp")] + [
    os.path.join(INCLUDE, f) for f in ("iwp_loss.h", "iwp.h")]
AROUND_DEPS = [os.path.join(CSRC, f) for f in ("iwp_route.cu", "iwp_route_f32.cu", "iwp_route_bf16.cu", "iwp_route_f16.cu", "iwp_route.cuh",
                                               "iwp_route_launch.hpp", "iwp_exchange.cuh", "iwp_clip.cu", "iwp_clip.cuh", "iwp_elem.cuh")] + [
    os.path.join(INCLUDE, f) for f in ("iwp_route.h", "iwp_clip.h")]
DEPS = STEP_DEPS + LOSS_DEPS + AROUND_DEPS

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC"]
# The step is bit-exact against its oracle: IEEE arithmetic, no FMA contraction, correctly rounded division, denormals
# kept.  The losses, the router and the clipping are held to tolerances and use the compiler's defaults.
SOURCES = [
    (os.path.join(CSRC, "iwp_api.cu"), ["-fmad=false", "-prec-div=true", "-prec-sqrt=true", "-ftz=false"]),
    (os.path.join(CSRC, "iwp_loss.cu"), []),
    (os.path.join(CSRC, "iwp_route.cu"), []),
    (os.path.join(CSRC, "iwp_route_f32.cu"), []),
    (os.path.join(CSRC, "iwp_route_bf16.cu"), []),
    (os.path.join(CSRC, "iwp_route_f16.cu"), []),
    (os.path.join(CSRC, "iwp_clip.cu"), []),
]


# The same library with every computed index of the step's kernels range-checked and the histogram counts checked for
# conservation (a failed check sets the status word; nothing traps), and with a kernel whose bounded waits run out, for the
# losses' tests.  The losses' kernels have no checks of their own.  Loaded instead of libiwp.so when IWP_LIB_VARIANT=debug.
LIB_DEBUG = os.path.join(HERE, "libiwp_debug.so")


def stale(lib: str = LIB) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    return any(os.path.getmtime(d) > t for d in DEPS)


def build(force: bool = False, verbose: bool = False, debug: bool = False) -> str:
    lib = LIB_DEBUG if debug else LIB
    if not force and not stale(lib):
        return lib
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    extra = (["-DIWP_DEBUG_CHECKS"] if debug else []) + (["-Xptxas", "-v"] if verbose else [])
    objects = [f"{lib}.{i}.o" for i in range(len(SOURCES))]
    steps = [[nvcc] + NVCC_FLAGS + flags + extra + ["-c", src, "-o", obj] for (src, flags), obj in zip(SOURCES, objects)]
    running = [subprocess.Popen(c, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True) for c in steps]
    outs = [p.communicate()[0] for p in running]
    ok = all(p.returncode == 0 for p in running)
    if ok:
        r = subprocess.run([nvcc] + NVCC_FLAGS + ["-shared"] + objects + ["-o", lib + ".tmp"], capture_output=True, text=True)
        outs.append(r.stdout + r.stderr)
        ok = r.returncode == 0
    for obj in objects:
        if os.path.exists(obj):
            os.remove(obj)
    if not ok:
        sys.stderr.write("".join(outs))
        raise RuntimeError(f"nvcc failed building {os.path.basename(lib)}")
    if verbose:
        sys.stderr.write("".join(outs))
    os.replace(lib + ".tmp", lib)
    return lib


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv, debug="--debug" in sys.argv))
