"""Register and spill budget of the kernels of a distillation step, read from ptxas at
build time, and that none touches memory before the kernel in front is done."""
import os
import re

import pytest

from paper_2512_09685_b200 import build

from .test_worker_step_launch_order import kernels
from .test_worker_step_resources import entries


@pytest.mark.parametrize("source,count", [("alternatives.cu", 14), ("distillation.cu", 26), ("norm.cu", 86)])
def test_kernels_fit(source, count):
    found = entries(source)
    assert len(found) == count, sorted(found)
    for name, r in found.items():
        few = 0
        m = re.search(r"star_distillation_kernelINS_\w+?ELi(\d+)", name)
        if m:                                            # 1024 threads an SM
            assert r["regs"] <= 64, (name, r)
            few = 128                                    # rows' scalars, outside the walks
        elif "star_alternatives_kernel" in name:         # 1280, or 1024
            assert r["regs"] <= 64, (name, r)
            few = 96
        elif "star_alternatives_backward" in name:       # 1280
            assert r["regs"] <= 48, (name, r)
        elif "rms_norm_backward_kernel" in name:         # 768 threads an SM in blocks of up to 256, or one larger block
            threads = int(re.search(r"ELb\dELi(\d+)E", name).group(1))
            assert r["regs"] <= {512: 128, 1024: 64}.get(threads, 85), (name, r)
            few = 128 if threads == 1024 else 48
        elif "ELi1024E" in name:                         # long rows in one block's registers
            few = 400
        assert r["spill"] <= few, (name, r)


@pytest.mark.parametrize("header", ["alternatives.cuh", "distillation.cuh", "norm.cuh"])
def test_memory_is_touched_after_the_wait(header):
    found = list(kernels(header))
    assert found
    for name, body in found:
        front = body[:body.index("wait_for_primary();")]
        front = front[front.index("{"):]
        assert not re.search(r"load_value|a\.(?!row\.inv_temperature|row\.vocab|row\.rows|rows|cols|k\b|gain\b)\w+", front), (name, front)
        assert "asm" not in front or "fence.mbarrier_init" in front or "mov" in front, name


def test_every_source_is_built():
    present = {f for f in os.listdir(build.CSRC) if f.endswith((".cu", ".cc"))}
    assert present == set(build.SOURCES)
    assert {os.path.basename(h) for h in build.HEADERS} >= {f for f in os.listdir(build.CSRC) if f.endswith((".cuh", ".h"))}
