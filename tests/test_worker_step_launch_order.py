"""The kernels of a worker's step may be set up while the kernel in front of them is
still running.  Until that one is done they must hold nothing that it may yet wait
for: accumulator memory is taken by an instruction that waits without limit, so it
comes after the wait for the kernel in front, which otherwise could wait for this one."""
import os
import re

import pytest

from paper_2512_09685_b200 import build


def kernels(header):
    text = open(os.path.join(build.CSRC, header)).read()
    starts = [m.start() for m in re.finditer(r"__global__", text)] + [len(text)]
    for a, b in zip(starts, starts[1:]):
        yield re.search(r"(star_\w+_kernel)\(", text[a:b]).group(1), text[a:b]


@pytest.mark.parametrize("header", ["losses.cuh", "checkpoint.cuh", "weight_grad.cuh"])
def test_accumulator_memory_is_taken_after_the_wait(header):
    found = list(kernels(header))
    assert found
    for name, body in found:
        wait = body.index("wait_for_primary();")
        assert "tensor_alloc<" not in body[:wait], name
