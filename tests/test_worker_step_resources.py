"""Register and spill budget of the kernels of a worker's step, read from ptxas
at build time: their launch shapes count on it."""
import os
import re
import subprocess

import pytest

from paper_2512_09685_b200 import build as lib_build


def entries(source):
    cmd = [lib_build.nvcc(), *lib_build.NVCC_FLAGS, "-I", os.path.join(lib_build.ROOT, "include"), "-I",
           lib_build.CSRC, "-Xptxas", "-v", os.path.join(lib_build.CSRC, source), "-o", os.devnull]
    out = subprocess.run(cmd, capture_output=True, text=True, timeout=900)
    assert out.returncode == 0, out.stderr[-2000:]
    found, current = {}, None
    for line in out.stderr.splitlines():
        m = re.search(r"Compiling entry function '(\S+)'", line)
        if m:
            current = m.group(1)
            found[current] = {"spill": None, "regs": None}
        elif current is not None:
            m = re.search(r"bytes stack frame, (\d+) bytes spill stores, (\d+) bytes spill loads", line)
            if m and found[current]["spill"] is None:
                found[current]["spill"] = int(m.group(1)) + int(m.group(2))
            m = re.search(r"Used (\d+) registers", line)
            if m:
                found[current]["regs"] = int(m.group(1))
    return found


@pytest.mark.parametrize("source,kernels", [("losses.cu", 37), ("checkpoint.cu", 48), ("weight_grad.cu", 18)])
def test_kernels_fit_and_do_not_spill(source, kernels):
    found = entries(source)
    assert len(found) == kernels, sorted(found)
    for name, r in found.items():
        m = re.search(r"star_policy_kernelINS_\w+?ELi(\d+)ELb(\d)E", name)
        if m:                                            # 1024 threads an SM
            assert r["regs"] <= 64, (name, r)
        elif "star_row_kernel" in name:                  # 1280
            assert r["regs"] <= 48 or "ELi32E" in name and r["regs"] <= 64, (name, r)
        elif "weight_grad_tensor" in name:               # 640 in a block
            assert r["regs"] <= 96, (name, r)
        # The rows' scalars of clusters, and the running sums' addresses: outside the inner loops.
        few = m and m.group(2) == "1" or "weight_grad_tensor" in name and "ELi0ELb1E" in name
        assert r["spill"] <= (192 if few else 0), (name, r)
