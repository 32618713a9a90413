"""The distillation loss where student and teacher nearly agree: how many digits a small
loss keeps."""
import pytest
import torch

from . import distillation_reference as R
from .test_gpu_distillation import BF16, F32, call, gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("temperature,k", [(1.0, 8), (1.0, 64), (2.0, 64), (4.0, 8)])
@pytest.mark.parametrize("noise", [1.0, 1e-1, 1e-2, 1e-3])
def test_errors_go_with_the_root_of_the_loss(noise, temperature, k, dtype):
    """With log ratios d, the loss is a sum of q d^2 / 2.  What all its logarithms share (the row's sum) cancels, for the
    sum of q d is that loss itself; what remains is the error of the rest's sum, at q0 |d0| <= sqrt(2 loss), and that of
    the terms, at the loss.  The rest's sum: 4 half steps for a power, one for each unit of an exponent (a mean of 8),
    8 for its additions; the terms a few half steps of d, whose share of d^2 / 2 is again one of d."""
    g = gpu(41)
    x = (torch.randn((16, 20011), generator=g, device="cuda") * 2).to(dtype)
    teacher = x.float() + noise * torch.randn(x.shape, generator=g, device="cuda")
    top, ids = torch.topk(teacher, k, 1)
    top = torch.log_softmax(teacher.double() / temperature, 1).gather(1, ids).float()
    more = dict(rest=True, temperature=temperature)
    loss, _, _ = call(x, ids.int(), top, out=None, **more)
    want = R.distillation(x, ids.int(), top, **more)["token_loss"]
    assert bool((want > 0).all())
    assert bool(((loss.double() - want).abs() <= 20 * R.ULP * (torch.sqrt(2 * want) + want)).all())
