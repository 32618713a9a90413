"""Labels whose logit is masked by the type's lowest value.  Formulas and tolerances are those of test_gpu_losses.py."""
import pytest
import torch

from tests import worker_step_reference as R
from tests.test_gpu_losses import GRAD, check_preference, close, make, policy_call, preference_call

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2512_09685_b200 import binding
    return binding


# rows of a block, read twice, read once, and kept by a cluster
SIZES = [(12, 300), (900, 1000), (1100, 1003), (1030, 30_000), (300, 120_001)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V", SIZES)
def test_a_label_masked_by_the_lowest_value(B, T, V, dtype):
    """Its log-probability is that value, which both types and the result hold, and not -inf: old and
    reference values of the same token cancel it."""
    lowest = torch.finfo(dtype).min
    x, labels, g = make(T, V, dtype, seed=V, masked=0.0)
    rows = torch.arange(1, T, 5, device="cuda")
    x[rows, labels[rows]] = lowest
    x[rows[::2], : V // 2] = lowest                        # and much else with it
    x[rows[::2], labels[rows[::2]]] = lowest
    want, want_lse, _, _ = R.rows(x, labels)
    assert float(want.min()) == lowest                     # the rest of the sum is far below its last bit
    lp, lse = torch.full((T,), 7.0, device="cuda"), torch.full((T,), 7.0, device="cuda")
    B.star_token_logprobs(x, labels, lp, lse)
    assert close(lp, want) and close(lse, want_lse)
    B.star_token_logprobs(x, labels, lp, lse, temperature=4.0)
    assert close(lp, R.rows(x, labels, None, 4.0)[0])
    A = torch.randn(T, generator=g, device="cuda")
    kept = want.float()
    got = policy_call(B, x, labels, A, old_logp=kept, ref_logp=kept, kl_coef=0.5)
    ref = R.policy(x, labels, A, old=kept, ref=kept, kl_coef=0.5)
    assert close(got["logp"], ref["logp"])
    # the last bits of the others' log-probabilities: kept to binary32, off by 4e-6 + 4e-7 of up to 15, twice
    assert close(got["token_loss"], ref["token_loss"], absolute=2e-5 * float(A.abs().max()))
    assert R.rel(got["dlogits"], ref["dlogits"]) <= GRAD[dtype] + 2e-5
    alone = policy_call(B, x, labels, A, dlogits=None, old_logp=kept, ref_logp=kept, kl_coef=0.5)
    assert torch.equal(alone["logp"], got["logp"]) and torch.equal(alone["sums"], got["sums"])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_preference_with_a_label_masked_by_the_lowest_value(B, dtype):
    lowest = torch.finfo(dtype).min
    x, labels, g = make(20, 500, dtype, seed=4, masked=0.0)
    x[3, labels[3]] = lowest
    x[12, labels[12]] = lowest
    offsets = [0, 5, 10, 15, 20]
    ref = torch.randn(4, generator=g, device="cuda")
    got = preference_call(B, x, labels, offsets, ref_logp=ref, beta=0.4)
    want = R.preference(x, labels, offsets, ref=ref, beta=0.4)
    assert close(got["seq_logp"], want["seq_logp"], absolute=1e-4) and float(want["seq_logp"].min()) == lowest
    check_preference(got, want, dtype, 0.4, 20)
