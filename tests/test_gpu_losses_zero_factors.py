"""Policy loss with a factor of 0 beside one beyond binary32.  Formulas and tolerances are those of test_gpu_losses.py."""
import math

import pytest
import torch

from tests import worker_step_reference as R
from tests.test_gpu_losses import GRAD, LOSS, close, make, policy_call

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2512_09685_b200 import binding
    return binding


# rows of a block, read twice, read once, and kept by a cluster
SIZES = [(12, 300), (900, 1000), (1100, 1003), (1030, 30_000), (300, 120_001)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V", SIZES)
def test_a_factor_of_zero_takes_its_term_out(B, T, V, dtype):
    """exp(100) is beyond binary32: times an advantage of 0, or a KL coefficient of 0, it is 0 all the same."""
    x, labels, g = make(T, V, dtype, seed=V + 1, masked=0.2)
    lp = R.rows(x, labels)[0].float()
    A = torch.randn(T, generator=g, device="cuda")
    far = torch.arange(T, device="cuda") % 3 == 1
    old = lp - 0.1 * torch.rand(T, generator=g, device="cuda")
    A[far], old[far] = 0.0, lp[far] - 100.0
    for clip_high in (0.2, math.inf):
        got, want = policy_call(B, x, labels, A, old_logp=old, clip_high=clip_high), R.policy(x, labels, A, old=old, clip_high=clip_high)
        assert close(got["token_loss"], want["token_loss"], absolute=LOSS * 4)
        assert close(got["sums"], want["sums"], absolute=LOSS * 4 * T)
        assert R.rel(got["dlogits"], want["dlogits"]) <= GRAD[dtype]
        assert bool((got["dlogits"][far] == 0).all())
    far_ref = torch.where(far, lp + 100.0, lp + 0.3)
    got, want = policy_call(B, x, labels, A, ref_logp=far_ref, kl_coef=0.0), R.policy(x, labels, A, ref=far_ref, kl_coef=0.0)
    assert close(got["token_loss"], want["token_loss"], absolute=LOSS * 4)
    assert close(got["sums"][[0, 1, 3]], want["sums"][[0, 1, 3]], absolute=LOSS * 4 * T)
    assert float(got["sums"][2]) == math.inf               # the KL itself: 2.7e43 a token
    assert R.rel(got["dlogits"], want["dlogits"]) <= GRAD[dtype]


def test_a_row_of_nan_shows_whatever_its_factors_are(B):
    x, labels, _ = make(6, 100, torch.float32, seed=1, masked=0.0)
    x[2, 50] = math.nan
    for kw in (dict(), dict(old_logp=torch.zeros(6, device="cuda"))):
        got = policy_call(B, x, labels, torch.zeros(6, device="cuda"), **kw)
        assert bool(torch.isnan(got["token_loss"][2])) and bool(torch.isnan(got["dlogits"][2]).all()) and bool(torch.isnan(got["sums"][0]))
        assert bool((got["dlogits"][[0, 1, 3, 4, 5]] == 0).all())
