"""The losses over the ranges of row counts at which the work is divided in
another way: clusters of blocks to a row, blocks of a warp with many rows, rows
read once or twice.  Plain implementation and tolerances are those of
test_gpu_losses.py."""
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


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V", [(64, 20_001), (149, 40_003), (290, 17_000), (300, 40_003), (600, 300), (1500, 5001), (1500, 20_001),
                                 (2100, 9000), (4800, 777), (9600, 100), (20_000, 33)])
def test_logprobs_over_numbers_of_rows(B, T, V, dtype):
    x, labels, _ = make(T, V, dtype, seed=V + T, masked=0.2)
    lp, lse = torch.full((T,), 7.0, device="cuda"), torch.full((T,), 7.0, device="cuda")
    B.star_token_logprobs(x, labels, lp, lse, temperature=0.7)
    want, want_lse, _, _ = R.rows(x, labels, None, 0.7)
    assert close(lp, want) and close(lse, want_lse)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 7, 9, 33, 255, 1025, 4096, 8191, 20_003, 57_344, 57_352, 70_001])
def test_policy_loss_of_rows_read_once(B, V, dtype):
    """Over the vocabulary sizes; the two longest rows are read twice in fp32, the last in both types."""
    T = 450 if V > 10_000 else 1000
    x, labels, g = make(T, V, dtype, seed=3 * V, masked=0.3)
    A = torch.randn(T, generator=g, device="cuda")
    w = torch.rand(T, generator=g, device="cuda") * (torch.rand(T, generator=g, device="cuda") < 0.9)
    ref = R.rows(x, labels)[0].float() + 0.5 * torch.randn(T, generator=g, device="cuda")
    kw = dict(weights=w, ref_logp=ref, kl_coef=0.3)
    got, want = policy_call(B, x, labels, A, **kw), R.policy(x, labels, A, weights=w, ref=ref, kl_coef=0.3)
    size = float((want["token_loss"].abs() + A.abs()).max())
    assert close(got["logp"], want["logp"])
    assert close(got["token_loss"], want["token_loss"], absolute=LOSS * max(size, 1.0))
    assert close(got["sums"], want["sums"], absolute=LOSS * T * max(size, 1.0))
    assert R.rel(got["dlogits"], want["dlogits"]) <= GRAD[dtype] or float(want["dlogits"].abs().max()) < 1e-6
    assert torch.equal(got["dlogits"][~want["active"]], torch.zeros_like(got["dlogits"][~want["active"]]))
    alone = policy_call(B, x, labels, A, dlogits=None, **kw)
    for name in ("logp", "token_loss", "sums"):
        assert torch.equal(alone[name], got[name]), name
    kept = x.clone()
    policy_call(B, x, labels, A, dlogits=x, **kw)
    assert torch.equal(x, got["dlogits"])
    assert V == 1 or not torch.equal(x, kept)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset,pad,out_offset,out_pad", [(1, 0, 1, 0), (1, 7, 5, 0), (3, 5, 0, 3), (0, 8, 0, 16), (2, 6, 4, 1)])
@pytest.mark.parametrize("V", [5, 40, 1003, 4096])
def test_strides_of_rows_read_once(B, V, offset, pad, out_offset, out_pad, dtype):
    T = 460
    x, labels, g = make(T, V, dtype, seed=V + offset, offset=offset, pad=pad)
    A = torch.randn(T, generator=g, device="cuda")
    ld = V + out_pad
    store = torch.full((out_offset + T * ld + 64,), 3.0, device="cuda").to(dtype)
    d = store[out_offset: out_offset + T * ld].view(T, ld)[:, :V]
    got, want = policy_call(B, x, labels, A, dlogits=d), R.policy(x, labels, A)
    assert close(got["logp"], want["logp"]) and R.rel(d, want["dlogits"]) <= GRAD[dtype]
    keep = torch.full_like(store, 3.0)
    keep[out_offset: out_offset + T * ld].view(T, ld)[:, :V] = d
    assert torch.equal(store.float(), keep.float())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_special_logits_of_rows_read_once(B, dtype):
    """Rows with nothing left, NaN, infinities and the type's lowest value, beside ordinary ones, which stay what they are alone."""
    T, V = 600, 1000
    x, labels, g = make(T, V, dtype, seed=9, masked=0.0)
    A = torch.randn(T, generator=g, device="cuda")
    old = R.rows(x, labels)[0].float()
    plain = policy_call(B, x, labels, A, old_logp=old)
    odd = torch.arange(3, T, 7, device="cuda")
    kinds = torch.arange(odd.numel(), device="cuda") % 6
    y = x.clone()
    y[odd[kinds == 0]] = -math.inf                        # nothing left: inactive
    y[odd[kinds == 1]] = torch.finfo(dtype).min           # uniform
    y[odd[kinds == 2], 500] = math.nan
    y[odd[kinds == 3], 10:] = -math.inf                   # the label masked as well
    marked = labels.clone()
    marked[odd[kinds == 3]] = 900
    y[odd[kinds == 4]] = math.nan                         # not read: the label leaves it out
    marked[odd[kinds == 4]] = -100
    y[odd[kinds == 5], 10:] = -math.inf
    marked[odd[kinds == 5]] = 4
    got, want = policy_call(B, y, marked, A, old_logp=old), R.policy(y, marked, A, old=old)
    rest = torch.ones(T, dtype=torch.bool, device="cuda")
    rest[odd] = False
    assert torch.equal(got["dlogits"][rest], plain["dlogits"][rest]) and torch.equal(got["logp"][rest], plain["logp"][rest])
    masked = want["logp"] == -math.inf
    assert torch.equal(got["logp"] == -math.inf, masked)
    assert close(got["logp"][~masked], want["logp"][~masked])
    for t in odd.tolist():
        w, h = want["dlogits"][t], got["dlogits"][t]
        assert bool(torch.isnan(w).any()) == bool(torch.isnan(h).any()), t
        if not bool(torch.isnan(w).any()):
            assert R.rel(h, w) <= GRAD[dtype] or float(w.abs().max()) < 1e-6, t


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V", [(1100, V) for V in (1, 2, 7, 9, 33, 255, 1025, 4096, 8191, 20_003)]
                         + [(1025, 3584), (1025, 28_672), (1030, 28_680), (300, 90_001), (130, 120_001), (64, 229_376), (64, 240_001)])
def test_policy_loss_of_many_or_long_rows(B, T, V, dtype):
    """Blocks of 32 threads to clusters of eight blocks of 512, and what is longer than those hold."""
    x, labels, g = make(T, V, dtype, seed=5 * V, offset=3, pad=1, masked=0.3)
    A = torch.randn(T, generator=g, device="cuda")
    old = R.rows(x, labels)[0].float()
    got, want = policy_call(B, x, labels, A, old_logp=old), R.policy(x, labels, A, old=old)
    size = float((want["token_loss"].abs() + A.abs()).max())
    assert close(got["logp"], want["logp"])
    assert close(got["token_loss"], want["token_loss"], absolute=LOSS * max(size, 1.0))
    assert close(got["sums"], want["sums"], absolute=LOSS * T * max(size, 1.0))
    assert R.rel(got["dlogits"], want["dlogits"]) <= GRAD[dtype] or float(want["dlogits"].abs().max()) < 1e-6
    assert torch.equal(got["dlogits"][~want["active"]], torch.zeros_like(got["dlogits"][~want["active"]]))
    del want
    alone = policy_call(B, x, labels, A, dlogits=None, old_logp=old)
    for name in ("logp", "token_loss", "sums"):
        assert torch.equal(alone[name], got[name]), name
    policy_call(B, x, labels, A, dlogits=x, old_logp=old)
    assert torch.equal(x, got["dlogits"])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset,pad,out_offset,out_pad", [(1, 0, 1, 0), (1, 7, 5, 0), (3, 5, 0, 3), (0, 8, 0, 16), (2, 6, 4, 1)])
@pytest.mark.parametrize("T,V", [(1030, 5), (1030, 40), (1030, 1003), (400, 60_001)])
def test_strides_of_many_or_long_rows(B, T, V, offset, pad, out_offset, out_pad, dtype):
    test_strides_of_rows(B, T, V, offset, pad, out_offset, out_pad, dtype)


def test_strides_of_rows(B, T=470, V=77, offset=1, pad=2, out_offset=3, out_pad=4, dtype=torch.bfloat16):
    x, labels, g = make(T, V, dtype, seed=V + offset, offset=offset, pad=pad)
    A = torch.randn(T, generator=g, device="cuda")
    ld = V + out_pad
    store = torch.full((out_offset + T * ld + 64,), 3.0, device="cuda").to(dtype)
    d = store[out_offset: out_offset + T * ld].view(T, ld)[:, :V]
    got, want = policy_call(B, x, labels, A, dlogits=d), R.policy(x, labels, A)
    assert close(got["logp"], want["logp"]) and R.rel(d, want["dlogits"]) <= GRAD[dtype]
    keep = torch.full_like(store, 3.0)
    keep[out_offset: out_offset + T * ld].view(T, ld)[:, :V] = d
    assert torch.equal(store.float(), keep.float())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V", [(1200, 1000), (400, 60_001)])
def test_special_logits_among_many_or_long_rows(B, T, V, dtype):
    x, labels, g = make(T, V, dtype, seed=9, masked=0.0)
    A = torch.randn(T, generator=g, device="cuda")
    old = R.rows(x, labels)[0].float()
    plain = policy_call(B, x, labels, A, old_logp=old)
    odd = torch.arange(3, T, 7, device="cuda")
    kinds = torch.arange(odd.numel(), device="cuda") % 6
    y, marked = x.clone(), labels.clone()
    y[odd[kinds == 0]] = -math.inf                        # nothing left: inactive
    y[odd[kinds == 1]] = torch.finfo(dtype).min           # uniform
    y[odd[kinds == 2], V // 2] = math.nan
    y[odd[kinds == 3], 10:] = -math.inf                   # the label masked as well
    marked[odd[kinds == 3]] = V - 100
    y[odd[kinds == 4]] = math.nan                         # not read: the label leaves it out
    marked[odd[kinds == 4]] = V
    y[odd[kinds == 5], : V - 10] = -math.inf              # only the end is left
    marked[odd[kinds == 5]] = V - 4
    got, want = policy_call(B, y, marked, A, old_logp=old), R.policy(y, marked, A, old=old)
    rest = torch.ones(T, dtype=torch.bool, device="cuda")
    rest[odd] = False
    assert torch.equal(got["dlogits"][rest], plain["dlogits"][rest]) and torch.equal(got["logp"][rest], plain["logp"][rest])
    none = want["logp"] == -math.inf
    assert torch.equal(got["logp"] == -math.inf, none) and close(got["logp"][~none], want["logp"][~none])
    for t in odd.tolist():
        w, h = want["dlogits"][t], got["dlogits"][t]
        assert bool(torch.isnan(w).any()) == bool(torch.isnan(h).any()), t
        if not bool(torch.isnan(w).any()):
            assert R.rel(h, w) <= GRAD[dtype] or float(w.abs().max()) < 1e-6, t
