"""Build the GoCkpt HIP library for gfx950 in-tree.

    python -m paper_2511_07035_amd.build

Produces ``paper_2511_07035_amd/libgockpt.so`` (the C-ABI declared in
``include/gockpt.h`` and ``include/gockpt_ops.h``) and ``paper_2511_07035_amd/libgockpt_bench.so`` (device
helpers of the benchmark harness and tests: the forward/backward stand-in,
HBM probes, a kernel that holds every wave slot, and a device division and
square root for bitwise checks).
Cross-compiles without a GPU.
"""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libgockpt.so")
BENCH_LIB = os.path.join(PKG, "libgockpt_bench.so")

ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
HIPCC = os.path.join(ROCM, "bin", "hipcc")
CLANGXX = os.path.join(ROCM, "llvm", "bin", "clang++")
ARCH = "gfx950"

# IEEE arithmetic contract: no contraction into FMA, no fast-math, correctly
# rounded fp32 division/sqrt (HIP's default), subnormals kept (default).
# Packed fp32 instructions are disabled for every device build.
HIP_FLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off", "-fno-math-errno",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Xarch_host", "-mavx2", "-Wall", "-Wno-unused-command-line-argument", f"-I{INCLUDE}",
]
HOST_FLAGS = ["-O3", "-std=c++17", "-fPIC", "-ffp-contract=off", "-fno-math-errno", "-mavx2", "-msse4.2", "-Wall",
              f"-I{INCLUDE}"]

LIB_HIP = ["gockpt_kernels.hip", "gockpt_cast.hip", "gockpt_runtime.hip", "gockpt_grads.hip", "gockpt_embed.hip"]
LIB_HOST = ["gockpt_plan.cpp", "gockpt_planner.cpp", "gockpt_restore.cpp", "gockpt_persist.cpp"]
BENCH_HIP = ["bench_kernels.hip"]


def _run(cmd):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError("build failed: " + " ".join(cmd))
    # hipcc's host pass does not know the packed-fp32 feature flag; drop that
    # harmless warning, keep the rest.
    noise = [ln for ln in (r.stdout + r.stderr).splitlines() if ln.strip() and "packed-fp32-ops" not in ln]
    if noise:
        sys.stderr.write("\n".join(noise) + "\n")


def _link(out, objs, tmp):
    part = out + ".tmp"
    _run([HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", part, *objs, "-lpthread"])
    os.replace(part, out)


def build(verbose: bool = False) -> None:
    with tempfile.TemporaryDirectory(prefix="gockpt_build_") as tmp:
        objs = []
        for src in LIB_HIP:
            o = os.path.join(tmp, src + ".o")
            _run([HIPCC, *HIP_FLAGS, "-c", os.path.join(CSRC, src), "-o", o])
            objs.append(o)
        for src in LIB_HOST:
            o = os.path.join(tmp, src + ".o")
            _run([CLANGXX, *HOST_FLAGS, "-c", os.path.join(CSRC, src), "-o", o])
            objs.append(o)
        _link(LIB, objs, tmp)
        bobjs = []
        for src in BENCH_HIP:
            o = os.path.join(tmp, src + ".o")
            _run([HIPCC, *HIP_FLAGS, "-c", os.path.join(CSRC, src), "-o", o])
            bobjs.append(o)
        _link(BENCH_LIB, bobjs, tmp)
    if verbose:
        print("built", LIB, BENCH_LIB)


if __name__ == "__main__":
    build(verbose=True)
