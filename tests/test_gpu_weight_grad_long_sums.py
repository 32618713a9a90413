"""Weight gradients over thousands of rows in one part, where what an accumulator
loses would show: several runs of the running sum, the lower terms of an fp32 dy.

Tolerance, set before the first run.  Products are exact.  The tensor cores' additions
cut: 1.2e-6 of a sum of one sign over a run of 1280 rows.  Runs are added with
rounding, at most 13 of them here: half a unit each at worst, 2e-7 as they come; the terms of an
fp32 dy hold all its bits, and their two accumulators are added once more, the lower
one of all rows with cuts of its own, 3e-7.  Below 2e-6 together, whatever the number of rows,
for random signs and for one sign.  Runs of 2048 rows are off by 2.3e-6 to 2.7e-6, one accumulator over
16384 rows by 1.9e-5, an fp32 dy without its third term by 4e-6 or more."""
import pytest
import torch

from tests import worker_step_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2512_09685_b200 import binding
    return binding


def case(B, T, C, O, dy_dtype, pad, one_sign, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((T, C), generator=g, device="cuda")
    dy = torch.randn((T, O + pad), generator=g, device="cuda")
    if one_sign:
        x, dy = x.abs_(), dy.abs_()
    dy = dy.to(dy_dtype)[:, :O]
    codes, scales = B.star_checkpoint_empty(T, C)
    B.star_checkpoint_pack(codes, scales, x)
    B.star_checkpoint_unpack(x, codes, scales)
    want = torch.zeros((O, C), dtype=torch.float64, device="cuda")
    for a in range(0, T, 2048):
        want += dy[a: a + 2048].double().t() @ x[a: a + 2048].double()
    return codes, scales, dy, want


# (columns, outputs): 64 tiles of a pair of blocks, and a number of columns that suits single blocks better, for the tiles
# of 256 and of 128 outputs.
@pytest.mark.parametrize("one_sign", [False, True])
@pytest.mark.parametrize("T,C,O,dy_dtype,pad", [
    (16384, 1024, 4096, torch.bfloat16, 0), (8192, 384, 11_520, torch.bfloat16, 0),
    (8192, 1024, 2048, torch.bfloat16, 1), (8192, 384, 5760, torch.bfloat16, 1),
    (16384, 1024, 2048, torch.float32, 0), (8192, 384, 5760, torch.float32, 0), (7001, 1000, 2040, torch.float32, 3)])
def test_fp32_sums_do_not_lose_with_their_length(B, T, C, O, dy_dtype, pad, one_sign):
    codes, scales, dy, want = case(B, T, C, O, dy_dtype, pad, one_sign, seed=C + O)
    dw = torch.full((O, C), 7.0, device="cuda")
    B.star_checkpoint_weight_grad(dw, dy, codes, scales)
    assert R.rel(dw, want) <= 2e-6
    B.star_checkpoint_weight_grad(dw, dy, codes, scales, accumulate=True)
    assert R.rel(dw, 2 * want) <= 2e-6
