"""Weight gradients of few rows: on both sides of where the tensor cores take over from the
ordinary units, at widths that fill whole tiles and others, in both layouts.  Plain
implementation and bounds are those of test_gpu_checkpoint.py."""
import pytest
import torch

from tests.test_gpu_checkpoint import weight_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2512_09685_b200 import binding
    return binding


@pytest.mark.parametrize("dy_dtype,dw_dtype", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32)])
@pytest.mark.parametrize("T", [1, 2, 3, 7, 8, 12, 16, 31, 32, 33, 48, 64])
def test_rows_on_both_sides(B, T, dy_dtype, dw_dtype):
    for C, O in ((256, 256), (1000, 1030), (1024, 2048)):
        weight_case(B, T, C, O, dy_dtype, dw_dtype, seed=T + C)
        weight_case(B, T, C, O, dy_dtype, dw_dtype, seed=T + C + 1, transposed=True, accumulate=True)


@pytest.mark.parametrize("T", [2, 8, 16, 40])
def test_a_large_result_from_few_rows(B, T):
    for dy_dtype, dw_dtype in ((torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32)):
        weight_case(B, T, 4096, 4100, dy_dtype, dw_dtype, seed=T, accumulate=True)
