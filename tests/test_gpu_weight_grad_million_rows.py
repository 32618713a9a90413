"""Weight gradients over more rows than one accumulator may take."""
import pytest
import torch

from tests import worker_step_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2512_09685_b200 import binding
    return binding


def test_a_bf16_result_over_a_million_rows_is_not_biased(B):
    """Sums of one sign whose sizes fill a binade: each result is rounded by up to 2^-9 of itself, at
    random, so that the mean over 65536 of them is off by 4.4e-6 (one standard deviation; 2e-5 is 4.5
    of them); the sums themselves add 2e-6.  Bound 3e-5.  One accumulator a part, of 300000 rows, is off by 1e-4 or more, all to one side."""
    T, C, O = 1_200_000, 128, 512
    g = torch.Generator(device="cuda").manual_seed(7)
    size = lambda n: torch.exp2(torch.rand(n, generator=g, device="cuda"))  # noqa: E731
    x = (0.5 + torch.rand((T, C), generator=g, device="cuda")) * size(C)
    dy = torch.empty((T, O), dtype=torch.bfloat16, device="cuda")
    sizes = size(O)
    for a in range(0, T, 100_000):
        dy[a: a + 100_000] = (0.5 + torch.rand((100_000, O), generator=g, device="cuda")) * sizes
    codes, scales = B.star_checkpoint_empty(T, C)
    B.star_checkpoint_pack(codes, scales, x)
    B.star_checkpoint_unpack(x, codes, scales)
    want = torch.zeros((O, C), dtype=torch.float64, device="cuda")
    for a in range(0, T, 50_000):
        want += dy[a: a + 50_000].double().t() @ x[a: a + 50_000].double()
    dw = torch.empty((O, C), dtype=torch.bfloat16, device="cuda")
    B.star_checkpoint_weight_grad(dw, dy, codes, scales)
    error = (dw.double() - want) / want
    assert float(error.abs().max()) <= 2.0 ** -8
    assert abs(float(error.mean())) <= 3e-5


def test_the_lower_terms_of_an_fp32_gradient_over_millions_of_rows(B):
    """The bound of some thousands of rows, 2e-6 (test_gpu_weight_grad_long_sums.py): the 240 runs of a part are
    added with rounding, 2e-7 as they come.  One accumulator for the lower terms of all 300000 rows of a part
    loses about 2e-3 of sums that are 2^-9 of the whole, 4e-6."""
    T, C, O = 2_400_000, 128, 128
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((T, C), generator=g, device="cuda").abs_()
    dy = torch.randn((T, O), generator=g, device="cuda").abs_()
    codes, scales = B.star_checkpoint_empty(T, C)
    B.star_checkpoint_pack(codes, scales, x)
    B.star_checkpoint_unpack(x, codes, scales)
    want = torch.zeros((O, C), dtype=torch.float64, device="cuda")
    for a in range(0, T, 100_000):
        want += dy[a: a + 100_000].double().t() @ x[a: a + 100_000].double()
    dw = torch.empty((O, C), device="cuda")
    B.star_checkpoint_weight_grad(dw, dy, codes, scales)
    assert R.rel(dw, want) <= 2e-6
