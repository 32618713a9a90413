"""Matrices that share rows of one buffer side by side: their address ranges meet,
their elements do not.  Formulas and tolerances are those of the operators' own tests."""
import pytest
import torch

from tests import worker_step_reference as R
from tests.test_gpu_checkpoint import ACT, keep, make as make_activations
from tests.test_gpu_losses import GRAD, close, make, policy_call, preference_call

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2512_09685_b200 import binding
    return binding


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V", [(5, 40), (1100, 1003)])
def test_losses_beside_their_gradient(B, T, V, dtype):
    x, labels, g = make(T, V, dtype, seed=V)
    both = torch.full((T, 2 * V + 3), 3.0, device="cuda").to(dtype)
    logits, d = both[:, V + 3:], both[:, 1: V + 1]
    logits.copy_(x)
    A = torch.randn(T, generator=g, device="cuda")
    same = both.clone()[:, V + 3:]                         # alone, at the same phases: the same bits
    got, want = policy_call(B, logits, labels, A, dlogits=d), R.policy(x, labels, A)
    assert close(got["logp"], want["logp"]) and R.rel(d, want["dlogits"]) <= GRAD[dtype]
    alone = d.clone()
    d.fill_(3.0)
    offsets = [0, T // 3, T]
    pref = preference_call(B, logits, labels, offsets, dlogits=d)
    apart = preference_call(B, same, labels, offsets)
    assert all(torch.equal(pref[n], apart[n]) for n in pref)
    assert torch.equal(logits, x) and bool((both[:, [0, V + 1, V + 2]] == 3.0).all())
    assert torch.equal(policy_call(B, same, labels, A)["dlogits"], alone)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("C", [64, 129])
def test_activations_beside_each_other(B, C, dtype):
    T = 70
    x, _ = make_activations(T, C, dtype, seed=C)
    dy, _ = make_activations(T, C, dtype, seed=C + 1)
    both = torch.full((T, 2 * C), 3.0, device="cuda").to(dtype)
    left, right = both[:, :C], both[:, C:]
    right.copy_(x)
    codes, scales = keep(B, right, act="gelu_tanh", act_out=left)
    assert R.rel(left, R.act(x.double(), "gelu_tanh")) <= ACT[dtype] and torch.equal(right, x)
    values = R.kept(x)[2]
    left.copy_(dy)
    B.star_checkpoint_act_backward(right, left, codes, scales, "silu")
    assert R.rel(right, dy.double() * R.act_slope(values, "silu")) <= ACT[dtype] and torch.equal(left, dy)


def test_what_does_overlap_is_refused(B):
    both = torch.zeros((8, 100), device="cuda")
    codes, scales = B.star_checkpoint_empty(8, 40)
    x = both[:, :40]
    # a column in common; one that wraps into the next row; the same columns a row further; strides that differ
    for other in (both[:, 39:79], both.reshape(-1)[61: 61 + 700].view(7, 100)[:, :40], both[1:, :40], both.reshape(-1)[50: 50 + 8 * 90].view(8, 90)[:, :40]):
        rows = min(other.shape[0], 8)
        c, s = (codes, scales) if rows == 8 else B.star_checkpoint_empty(rows, 40)
        before = B.star_launch_count()
        with pytest.raises(B.StarError) as e:
            B.star_checkpoint_pack(c, s, x[:rows], act="silu", act_out=other)
        assert e.value.status == B.STAR_ERR_INVALID_ARG and B.star_launch_count() == before
