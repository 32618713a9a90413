"""Build step: compiles the CUDA library in-tree with nvcc for sm_100a.

    python -m paper_2512_09685_b200.build

produces ``paper_2512_09685_b200/libstar.so`` from ``csrc/``.  nvcc
cross-compiles without a GPU.  The CUDA runtime is linked statically, so the
library depends on the driver only.
"""
from __future__ import annotations

import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libstar.so")
SOURCES = ["api.cu", "losses.cu", "alternatives.cu", "distillation.cu", "norm.cu", "checkpoint.cu", "weight_grad.cu", "schedule.cc",
           "mode_decision.cc"]
HEADERS = [os.path.join(CSRC, h) for h in ("internal.h", "kernels.cuh", "device.cuh", "rows.cuh", "rows_host.h", "losses.cuh",
                                           "alternatives.cuh", "distillation.cuh", "norm.cuh", "checkpoint.cuh",
                                           "checkpoint_host.h", "weight_grad.cuh")]
HEADERS.append(os.path.join(ROOT, "include", "star.h"))

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a",
    "-O3", "-std=c++17", "-lineinfo",
    "-fmad=false",                 # no implicit contraction: every FMA in the source is explicit
    "-Xcompiler", "-fPIC,-fvisibility=hidden,-Wall",
    "-shared", "-cudart", "static",
]


def nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    raise RuntimeError("nvcc not found")


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    built = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, s) for s in SOURCES] + HEADERS + [os.path.abspath(__file__)]
    return any(os.path.getmtime(d) > built for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not is_stale():
        return LIB
    tmp = LIB + ".tmp.%d" % os.getpid()
    cmd = [nvcc(), *NVCC_FLAGS, "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [os.path.join(CSRC, s) for s in SOURCES] + ["-o", tmp]
    subprocess.check_call(cmd)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
