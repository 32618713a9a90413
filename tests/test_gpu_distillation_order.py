"""The distillation loss over enough logits, some of whose rows take no part, that its rows
are taken in an order of their own (from 200 MB on, four rows to a block or cluster, up to
65536 of them): every row against calls of parts too small for that, bit for bit."""
import math

import pytest
import torch

from . import distillation_reference as R
from .test_gpu_distillation import BF16, F32, call, gpu, make, near
from .test_gpu_distillation_clusters import laid_out

pytestmark = pytest.mark.gpu


def masked(kind, rows, vocab, labels, w):
    drop = torch.rand(rows, generator=gpu(21), device="cuda") < 0.4
    if kind == "labels":
        labels[drop] = -100
    elif kind == "weights":
        w[drop] = 0.0
    elif kind == "all":
        w += 1.0
    elif kind == "none":
        w[:] = 0.0
    elif kind == "one":
        labels[:] = -1
        labels[rows // 2] = 7
    elif kind == "last":
        labels[:-3] = vocab
    else:
        labels[rows // 60:rows * 2 // 3] = vocab
    return (labels < 0) | (labels >= vocab) | (w == 0)


@pytest.mark.parametrize("kind", ["labels", "weights", "all", "none", "one", "last", "runs"])
@pytest.mark.parametrize("rows,vocab,dtype", [(6007, 20011, BF16), (6007, 10007, F32), (1500, 70001, BF16), (65536, 1609, BF16), (65537, 1609, BF16)])
def test_rows_in_an_order_of_their_own(rows, vocab, dtype, kind):
    assert rows * vocab * (2 if dtype is BF16 else 4) >= 200_000_000
    ld = (vocab + 16) // 8 * 8                           # all rows at one phase of the 16-byte grid
    x, ids, values, labels, w = make(rows, vocab, 9, dtype, seed=20, rest=True, ld=ld, offset=3)
    off = masked(kind, rows, vocab, labels, w)
    x[off] = math.nan
    values[off] = math.nan
    more = dict(rest=True, label_coef=0.5, temperature=1.3)
    out = laid_out(rows, vocab, ld, dtype)
    loss, sums, dx = call(x, ids, values, out=out, labels=labels, weights=w, **more)
    half = rows // 2
    for part in (slice(0, half), slice(half, rows)):
        n = part.stop - part.start
        assert n * vocab * x.element_size() < 200_000_000
        apart = call(x[part], ids[part], values[part], out=laid_out(n, vocab, ld, dtype), labels=labels[part], weights=w[part], **more)
        assert torch.equal(loss[part], apart[0]) and torch.equal(dx[part], apart[2])
    assert bool((loss[off] == 0).all()) and bool((dx[off] == 0).all())
    on = torch.nonzero(~off)[:, 0]
    pick = on[torch.randperm(len(on), generator=gpu(22), device="cuda")[:12]]
    if len(pick):
        want = R.distillation(x[pick], ids[pick], values[pick], labels=labels[pick], weights=w[pick], temperature=1.3, rest=True, hard=0.5)
        near(loss[pick], want["token_loss"], want["token_bound"])
        near(dx[pick], want["dlogits"], want["grad_bound"] + R.half_step(dtype) * want["dlogits"].abs())
    total = torch.where(off, torch.zeros_like(w), w).double()
    assert abs(float(sums[0]) - float((total * loss.double()).sum())) <= 8 * R.ULP * float((total * loss.double().abs()).sum())
    assert abs(float(sums[3]) - float(total.sum())) <= 8 * R.ULP * float(total.sum())
    again = call(x, ids, values, in_place=True, labels=labels, weights=w, **more)
    assert torch.equal(again[0], loss) and torch.equal(again[1], sums) and torch.equal(again[2], dx)
