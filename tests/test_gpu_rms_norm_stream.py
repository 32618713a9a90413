"""The stream that the residual norm leaves behind: x + residual, rounded once, to the bit."""
import math

import pytest
import torch

from .test_gpu_rms_norm import BF16, F32, SIZES, matrix

pytestmark = pytest.mark.gpu


def bits(x):
    return torch.where(torch.isnan(x), torch.full_like(x, math.nan), x).contiguous().view(torch.int16 if x.dtype is BF16 else torch.int32)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("offset,extra", [(0, 0), (1, 0), (5, 3), (8, 8)])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_total(rows, cols, offset, extra, dtype):
    from paper_2512_09685_b200 import binding as B
    x, res = matrix(rows, cols, dtype, 1, cols + extra, offset), matrix(rows, cols, dtype, 2, cols + extra, offset)
    x[-1, cols // 2], res[0, -1], x[0, 0] = math.nan, math.inf, -0.0
    for residual in (res, None):
        want = x.clone() if residual is None else (x.float() + residual.float()).to(dtype)
        total = matrix(rows, cols, dtype, 3, cols + extra, offset)
        B.star_rms_norm(torch.empty_like(x), x, residual=residual, total=total)
        assert torch.equal(bits(total), bits(want))
    place = res.clone() if extra == 0 and offset == 0 else res
    want = (x.float() + place.float()).to(dtype)
    B.star_rms_norm(torch.empty_like(x), x, residual=place, total=place)
    assert torch.equal(bits(place), bits(want))
