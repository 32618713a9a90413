"""The distillation loss by clusters of blocks with several rows each, some of which take
no part: every row against the same rows without the others in between, bit for bit, and
a few of them against the formula in binary64."""
import math

import pytest
import torch

from . import distillation_reference as R
from .test_gpu_distillation import BF16, F32, call, gpu, make, near

pytestmark = pytest.mark.gpu


def dropped(kind, rows):
    if kind == "random":
        return torch.rand(rows, generator=gpu(31), device="cuda") < 0.5
    t = torch.arange(rows, device="cuda")
    return (t // 37) % 2 == 0 if kind == "runs" else t % 3 == 1


def laid_out(rows, vocab, ld, dtype):
    return torch.full((3 + rows * ld,), 5.0, dtype=dtype, device="cuda")[3:].view(rows, ld)[:, :vocab]


@pytest.mark.parametrize("kind", ["random", "runs", "thirds"])
@pytest.mark.parametrize("rows,vocab,dtype", [(700, 128256, BF16), (1000, 70001, BF16), (800, 50257, F32), (600, 32001, F32)])
def test_clusters_of_several_rows_of_which_some_take_part(rows, vocab, dtype, kind):
    ld = (vocab + 16) // 8 * 8                           # all rows at one phase of the 16-byte grid
    x, ids, values, labels, w = make(rows, vocab, 24, dtype, seed=vocab, rest=True, ld=ld, offset=3)
    off = dropped(kind, rows)
    if kind == "thirds":
        w[off] = 0.0
    else:
        labels[off] = -100
    on = torch.nonzero(~off)[:, 0]
    more = dict(rest=True, soft_coef=0.5, label_coef=0.5)
    # Without the others in between.  As many threads and blocks to a row: more rows than would fill the GPU with more.
    less = laid_out(len(on), vocab, ld, dtype)
    less.copy_(x[on])
    alone = call(less, ids[on], values[on], out=laid_out(len(on), vocab, ld, dtype), labels=labels[on], weights=w[on], **more)
    out = laid_out(rows, vocab, ld, dtype)
    x[off] = math.nan
    values[off] = math.nan
    pick = on[torch.randperm(len(on), generator=gpu(32), device="cuda")[:12]]
    want = R.distillation(x[pick], ids[pick], values[pick], rest=True, labels=labels[pick], weights=w[pick], soft=0.5, hard=0.5)
    for in_place in (False, True):
        loss, sums, dx = call(x, ids, values, in_place=in_place, out=out, labels=labels, weights=w, **more)
        assert torch.equal(loss[on], alone[0]) and torch.equal(dx[on], alone[2])
        assert float(loss[off].abs().max()) == 0.0 and float(dx[off].abs().max()) == 0.0
        near(loss[pick], want["token_loss"], want["token_bound"])
        near(dx[pick], want["dlogits"], want["grad_bound"] + R.half_step(dtype) * want["dlogits"].abs())
        total = w[on].double()
        assert abs(float(sums[0]) - float((total * loss[on].double()).sum())) <= 8 * R.ULP * float((total * loss[on].double().abs()).sum())
        assert abs(float(sums[3]) - float(total.sum())) <= 8 * R.ULP * float(total.sum())


def test_a_wait_that_runs_out_between_rows_that_take_no_part():
    from paper_2512_09685_b200 import binding as B
    x, ids, values, labels, w = make(600, 32001, 8, F32, seed=33)
    labels[dropped("random", 600)] = -1
    B.star_check_waits()
    B.star_set_wait_attempts(0)
    try:
        sums = torch.zeros(4, device="cuda")
        ws = torch.empty(B.star_loss_workspace_bytes(600), dtype=torch.uint8, device="cuda")
        B.star_distillation_loss(x, ids, values, torch.zeros(600, device="cuda"), sums, ws, dlogits=torch.empty_like(x), labels=labels, weights=w)
        with pytest.raises(B.StarError) as e:
            B.star_check_waits()
        assert e.value.status == B.STAR_ERR_TIMEOUT
        assert bool(torch.isnan(sums).all())
    finally:
        B.star_set_wait_attempts()
    loss, _, _ = call(x, ids, values, labels=labels, weights=w)
    assert bool(torch.isfinite(loss).all())
