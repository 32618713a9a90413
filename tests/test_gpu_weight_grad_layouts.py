"""Both layouts of dw, written and added to, where the results go out by whole
sectors, by fours and by ones, from one block and from blocks that share the rows.
Plain implementation and bounds are those of test_gpu_checkpoint.py."""
import pytest
import torch

from tests.test_gpu_checkpoint import weight_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2512_09685_b200 import binding
    return binding


@pytest.mark.parametrize("dw_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dy_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("transposed,accumulate", [(False, True), (True, False), (True, True)])
@pytest.mark.parametrize("T,C,O", [(200, 640, 1024), (515, 256, 512), (2048, 1024, 1024), (1500, 300, 264), (3000, 130, 516), (2100, 2048, 4096)])
def test_weight_grad_layouts(B, T, C, O, transposed, accumulate, dy_dtype, dw_dtype):
    weight_case(B, T, C, O, dy_dtype, dw_dtype, seed=T, transposed=transposed, accumulate=accumulate)


@pytest.mark.parametrize("dw_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dw_offset,dw_pad", [(16, 16), (8, 8), (4, 4), (2, 6), (1, 0), (0, 1)])
def test_weight_grad_layouts_off_the_sectors(B, dw_offset, dw_pad, transposed, dw_dtype):
    for T, C, O in ((130, 256, 512), (1300, 256, 256)):
        weight_case(B, T, C, O, torch.bfloat16, dw_dtype, seed=T, dw_offset=dw_offset, dw_pad=dw_pad, transposed=transposed, accumulate=True)
