"""Rows of the residual norm that no block's registers hold: sums over them of one sign,
whose rounding does not average out."""
import pytest
import torch

from . import distillation_reference as R
from .test_gpu_rms_norm import BF16, F32, gpu, near

pytestmark = pytest.mark.gpu
# Sums of one sign: runs of 16 in binary32, a half step for each of their additions and products.
SUM = 16 * R.ULP


def one_sign(cols, value, dtype):
    """Two rows: one value throughout, and random ones of a sign."""
    x = torch.full((2, cols), value, device="cuda")
    x[1] = torch.rand(cols, generator=gpu(cols), device="cuda") + 0.5
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols,value", [(16385, 0.1), (70001, 0.3), (1 << 20, 0.1), (1 << 20, 0.3), (1 << 20, 3.7), ((1 << 22) + 5, 1.1)])
def test_sums_of_one_sign(cols, value, dtype):
    from paper_2512_09685_b200 import binding as B
    x = one_sign(cols, value, dtype)
    y, rstd = torch.empty_like(x), torch.empty(2, device="cuda")
    B.star_rms_norm(y, x, rstd=rstd, eps=1e-5)
    want, r = R.norm(x, None, 1e-5)
    # rstd by half of the sum's, and its own rounding; y by two more products' with the second number of rstd.
    near(rstd, r, (SUM / 2 + R.ULP) * r)
    near(y, want, (SUM / 2 + 2 * R.ULP + R.half_step(dtype)) * want)

    dy = one_sign(cols, 0.7 * value, dtype)
    dx = torch.empty_like(x)
    B.star_rms_norm_backward(dx, None, dy, None, rstd, total=x)
    want, _, _, _ = R.norm_backward(dy, x, rstd)
    n = x.double() * rstd.double()[:, None]
    mean = (dy.double() * n).mean(1, keepdim=True)
    # n, the sum, the mean and the difference are rounded once each, then dx.
    bound = rstd.double()[:, None] * n * mean * (SUM + 4 * R.ULP) + R.half_step(dtype) * want.abs() + R.ULP * want.abs()
    near(dx, want, bound)


def test_the_most_columns():
    """Rows that are 0 but at their ends, whose sums are exact: every column's index counts."""
    from paper_2512_09685_b200 import binding as B
    cols, ends = (1 << 31) - 65, 5000
    at = torch.cat([torch.arange(ends, device="cuda"), torch.arange(cols - ends, cols, device="cuda")])

    def row(seed):
        v = torch.randint(1, 17, (2 * ends,), generator=gpu(seed), device="cuda").to(BF16)
        x = torch.zeros((1, cols), dtype=BF16, device="cuda")
        x[0, at] = v
        return x, v.double()

    x, v = row(1)
    y, rstd = torch.full_like(x, 5.0), torch.empty(1, device="cuda")
    codes, scales = B.star_checkpoint_empty(1, cols)
    B.star_rms_norm(y, x, rstd=rstd, codes=codes, scales=scales, eps=1e-5)
    r = ((v * v).sum() / cols + 1e-5) ** -0.5
    near(rstd, r[None], R.ULP * r[None])
    near(y[0, at], v * r, (2 * R.ULP + R.half_step(BF16)) * v * r)
    assert int(torch.count_nonzero(y)) == 2 * ends
    again = B.star_checkpoint_empty(1, cols)
    B.star_checkpoint_pack(*again, y)
    assert torch.equal(codes, again[0]) and torch.equal(scales[:, 0], again[1][:, 0])
    del y, codes, scales, again

    dy, d = row(2)
    dx, dgain = torch.full_like(x, 5.0), torch.full((cols,), 5.0, device="cuda")
    ws = torch.empty(B.star_rms_norm_workspace_bytes(1, cols), dtype=torch.uint8, device="cuda")
    B.star_rms_norm_backward(dx, dgain, dy, None, rstd, ws, total=x)
    r = rstd.double()
    n = v * r
    near(dgain[at], d * n, 3 * R.ULP * d * n)
    want = r * (d - n * (d * n).sum() / cols)
    near(dx[0, at], want, R.half_step(BF16) * want.abs() + r * n * (d * n).sum() / cols * (SUM + 4 * R.ULP) + R.ULP * want.abs())
    assert int(torch.count_nonzero(dgain)) == 2 * ends and int(torch.count_nonzero(dx[:, ends:cols - ends])) == 0
