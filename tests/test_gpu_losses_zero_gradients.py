"""Active rows whose gradient is zero: every element of the output is written, and is zero."""
import math

import pytest
import torch

from tests.test_gpu_losses import make, policy_call, preference_call

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2512_09685_b200 import binding
    return binding


# rows of a block, read twice, read once (by the warp and by the block), and kept by a cluster
SIZES = [(5, 9), (40, 1003), (700, 4096), (1100, 1003), (1500, 9000), (300, 120_001)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [3, 1000, 1100])
def test_a_vocabulary_of_one(B, T, dtype):
    """p = 1 and the label is the only element: onehot - p = 0, exactly (2^0 / 1)."""
    x, labels, g = make(T, 1, dtype, seed=T, masked=0.2)
    A = 100 * torch.randn(T, generator=g, device="cuda")
    ref = torch.randn(T, generator=g, device="cuda")
    got = policy_call(B, x, labels, A, ref_logp=ref, kl_coef=0.5)
    assert bool((got["dlogits"] == 0).all()) and bool((got["logp"] == 0).all())
    got = preference_call(B, x, labels, [0, T // 2, T], beta=3.0)
    assert bool((got["dlogits"] == 0).all()) and bool((got["seq_logp"] == 0).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V", SIZES)
def test_rows_that_are_clipped_or_certain(B, T, V, dtype):
    x, labels, g = make(T, V, dtype, seed=V, masked=0.2)
    A = 1 + 10 * torch.rand(T, generator=g, device="cuda")
    certain = torch.arange(T, device="cuda") % 2 == 0
    at = labels.clamp(0, V - 1)
    alone = torch.full_like(x, -math.inf).scatter_(1, at[:, None], x.gather(1, at[:, None]))
    x[certain] = alone[certain]
    # the certain rows' gradient vanishes with onehot - p, the others' with a ratio e above the clip
    old = torch.full((T,), -1e3, device="cuda")
    old[certain] = 0.3
    d = torch.full((T, V + 5), 7.0, device="cuda").to(dtype)
    for out in ("new", d[:, :V], d[:, 3: V + 3]):          # the phases of the logits and others
        got = policy_call(B, x, labels, A, dlogits=out, old_logp=old)
        assert bool((got["dlogits"] == 0).all())
        d.fill_(7.0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V", SIZES)
def test_sequences_of_nothing_and_rows_of_none(B, T, V, dtype):
    x, labels, _ = make(T, V, dtype, seed=V)
    for offsets in ([0, 0, 0], [T, T, T], [2, 2, 2, 2, 2], [0]):
        got = preference_call(B, x, labels, offsets)
        assert bool((got["dlogits"] == 0).all())
    got = preference_call(B, x, labels, [1, 3, 4])
    assert bool((got["dlogits"][4:] == 0).all()) and bool((got["dlogits"][:1] == 0).all())
    assert V == 1 or bool((got["dlogits"][1:4][(labels[1:4] >= 0) & (labels[1:4] < V)] != 0).any(1).all())


@pytest.mark.parametrize("T,V", SIZES)
def test_no_scale_no_gradient(B, T, V):
    x, labels, g = make(T, V, torch.bfloat16, seed=V)
    got = preference_call(B, x, labels, [0, T // 2, T], loss_scale=0.0)
    assert bool((got["dlogits"] == 0).all()) and bool((got["loss"] == 0).all())
    got = policy_call(B, x, labels, torch.zeros(T, device="cuda"))
    assert bool((got["dlogits"] == 0).all()) and bool((got["token_loss"] == 0).all())
