"""Waits inside kernels that run out: with no attempts every wait has run out at
once, whatever the hardware does.  The kernels end, star_check_waits says so once,
nothing is written outside the outputs, and the next call is whole again."""
import math

import pytest
import torch

from paper_2512_09685_b200 import binding as B
from tests import worker_step_reference as R
from tests.test_gpu_losses import GRAD, make, policy_call


def test_attempts_are_checked():
    with pytest.raises(B.StarError) as e:
        B.star_set_wait_attempts(-1)
    assert e.value.status == B.STAR_ERR_INVALID_ARG
    B.star_set_wait_attempts(5)
    B.star_set_wait_attempts(2 ** 31 - 1)
    B.star_set_wait_attempts()


@pytest.fixture
def no_attempts():
    """Calls made inside it find every wait run out."""
    B.star_check_waits()

    class Attempts:
        def __enter__(self):
            B.star_set_wait_attempts(0)

        def __exit__(self, *_):
            B.star_set_wait_attempts()

    yield Attempts()
    B.star_set_wait_attempts()


def reported_once():
    with pytest.raises(B.StarError) as e:
        B.star_check_waits()
    assert e.value.status == B.STAR_ERR_TIMEOUT
    B.star_check_waits()


# Rows kept by blocks of 32, 128, 512 threads, by clusters of four and eight blocks; one row to a block and several.
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V", [(1100, 33), (3000, 1025), (1500, 8191), (500, 57_344), (300, 120_001), (130, 229_376)])
@pytest.mark.parametrize("grad", [True, False])
def test_policy_loss(no_attempts, T, V, dtype, grad):
    x, labels, g = make(T, V, dtype, seed=V, offset=3, pad=1, masked=0.3)
    A = torch.randn(T, generator=g, device="cuda")
    with no_attempts:
        got = policy_call(B, x, labels, A, dlogits="new" if grad else None)
    once = T * V * x.element_size() > 45_000_000 or T > 1024             # rows read twice do not wait
    if not once or V * x.element_size() > 224 * 512 * 8:
        B.star_check_waits()
        return
    assert bool(torch.isnan(got["sums"]).all())
    reported_once()
    # No row that is read has results; blocks may have gone past rows that are not.
    active = (labels >= 0) & (labels < V)
    assert bool((got["logp"][active] == 7.0).all()) and bool((got["token_loss"][active] == 7.0).all())
    if grad:
        assert bool((got["dlogits"][active] == 7.0).all())
    whole = policy_call(B, x, labels, A)
    want = R.policy(x, labels, A)
    assert R.rel(whole["dlogits"], want["dlogits"]) <= GRAD[dtype] and math.isfinite(float(whole["sums"][0]))
    B.star_check_waits()


# dy and dw in both types, dy on and off the 16-byte grid, one to many steps, parts of the rows, several runs of the running sum.
@pytest.mark.gpu
@pytest.mark.parametrize("dy_dtype,dw_dtype,pad", [(torch.bfloat16, torch.bfloat16, 0), (torch.bfloat16, torch.float32, 0),
                                                   (torch.bfloat16, torch.bfloat16, 1), (torch.float32, torch.float32, 0)])
@pytest.mark.parametrize("T,C,O", [(70, 256, 256), (515, 1024, 1024), (5000, 2048, 4096), (9000, 128, 128), (2500, 300, 264)])
def test_weight_grad(no_attempts, T, C, O, dy_dtype, dw_dtype, pad):
    g = torch.Generator(device="cuda").manual_seed(T)
    codes, scales = B.star_checkpoint_empty(T, C)
    B.star_checkpoint_pack(codes, scales, torch.randn((T, C), generator=g, device="cuda"))
    values = torch.empty((T, C), device="cuda")
    B.star_checkpoint_unpack(values, codes, scales)
    dy = torch.randn((T, O + pad), generator=g, device="cuda").to(dy_dtype)[:, :O]
    store = torch.full((O * C + 64,), 7.0, device="cuda").to(dw_dtype)
    dw = store[:O * C].view(O, C)
    with no_attempts:
        B.star_checkpoint_weight_grad(dw, dy, codes, scales)
        torch.cuda.synchronize()
    reported_once()
    assert bool((store == 7.0).all())
    B.star_checkpoint_weight_grad(dw, dy, codes, scales)
    B.star_check_waits()
    assert R.rel(dw, dy.double().t() @ values.double()) <= (4e-3 if dw_dtype == torch.bfloat16 else 1e-5)
    assert bool((store[O * C:] == 7.0).all())
