"""The policy loss with advantages of 1 and nothing else is the weighted
cross-entropy's gradient; its terms are the log-probabilities.  Tolerances are those
of test_gpu_losses.py."""
import pytest
import torch

from tests import worker_step_reference as R
from tests.test_gpu_losses import GRAD, close, make, policy_call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V", [(7, 101), (1100, 2003)])
def test_cross_entropy(T, V, dtype):
    from paper_2512_09685_b200 import binding as B
    x, labels, g = make(T, V, dtype, seed=V)
    w = torch.rand(T, generator=g, device="cuda")
    got = policy_call(B, x, labels, torch.ones(T, device="cuda"), weights=w, temperature=1.3)
    z = x.double().requires_grad_(True)
    target = torch.where((labels >= 0) & (labels < V), labels, -100)
    each = torch.nn.functional.cross_entropy(z / 1.3, target, ignore_index=-100, reduction="none")
    (w.double() * each).sum().backward()
    assert close(got["logp"], -each.detach()) and R.rel(got["dlogits"], z.grad) <= GRAD[dtype]
