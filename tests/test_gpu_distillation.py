"""The distillation loss and its gradient against the formulas in binary64.  Bounds
count half steps of binary32 (and the one rounding to bf16 of the gradient)."""
import math

import pytest
import torch

from . import distillation_reference as R

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def gpu(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def make(rows, vocab, k, dtype, seed=0, rest=False, noise=0.7, ld=None, offset=0, temperature=1.0):
    """A student's logits, and a teacher's list that differs from them by noise."""
    g = gpu(seed)
    ld = ld or vocab
    store = torch.zeros(offset + rows * ld + 64, dtype=dtype, device="cuda")
    x = store[offset:offset + rows * ld].view(rows, ld)[:, :vocab]
    x.copy_(torch.randn((rows, vocab), generator=g, device="cuda") * 2)
    t = x.float() + noise * torch.randn((rows, vocab), generator=g, device="cuda")
    if rest:
        t = torch.log_softmax(t / temperature, 1)
    n = min(k, vocab)
    values, ids = torch.topk(t, n, 1)
    wide_ids = torch.full((rows, k), -1, dtype=torch.int32, device="cuda")
    wide = torch.full((rows, k), -math.inf, device="cuda")
    wide_ids[:, :n], wide[:, :n] = ids.int(), values
    return x, wide_ids, wide, torch.randint(0, vocab, (rows,), generator=g, device="cuda"), torch.rand(rows, generator=g, device="cuda") + 0.5


def call(x, ids, values, in_place=False, out="own", **more):
    from paper_2512_09685_b200 import binding as B
    rows = x.shape[0]
    loss, sums = torch.full((rows,), 77.0, device="cuda"), torch.full((4,), 77.0, device="cuda")
    ws = torch.empty(B.star_loss_workspace_bytes(rows), dtype=torch.uint8, device="cuda")
    dx = None if out is None else x if in_place else torch.full_like(x, 5.0) if isinstance(out, str) else out
    B.star_distillation_loss(x, ids, values, loss, sums, ws, dlogits=dx, **more)
    B.star_check_waits()
    return loss, sums, dx


def check(x, ids, values, **more):
    kept = {n: more[n] for n in ("in_place", "out") if n in more}
    plain = {n: v for n, v in more.items() if n not in kept}
    names = {"soft_coef": "soft", "label_coef": "hard"}
    want = R.distillation(x, ids, values, **{names.get(n, n): v for n, v in plain.items()})
    loss, sums, dx = call(x, ids, values, **more)
    near(loss, want["token_loss"], want["token_bound"])
    near(sums, want["sums"], want["sums_bound"])
    if dx is not None:
        near(dx, want["dlogits"], want["grad_bound"] + R.half_step(x.dtype) * want["dlogits"].abs())
    return loss, sums, dx, want


def near(got, want, bound):
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), (got, want)
    far = torch.isinf(want)
    assert torch.equal(got[far], want[far])
    fine = torch.isfinite(want)
    off = (got - want).abs()[fine]
    assert bool((off <= bound[fine]).all()), float((off / bound[fine]).max())


SIZES = [(1, 1, 1, F32), (3, 5, 8, BF16), (1, 50257, 20, BF16), (5, 50257, 64, BF16), (7, 32001, 8, F32), (4, 2000, 128, BF16), (4, 1000, 128, F32),
         (50, 129, 3, BF16), (40, 257, 17, F32), (9, 4097, 1, BF16), (3, 64, 0, F32), (90, 3001, 33, BF16), (2, 131072, 40, F32), (3, 200000, 64, BF16)]


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,vocab,k,dtype", SIZES)
def test_sizes(rows, vocab, k, dtype, rest):
    x, ids, values, labels, w = make(rows, vocab, k, dtype, seed=rows + vocab, rest=rest)
    check(x, ids, values, rest=rest)
    check(x, ids, values, rest=rest, labels=labels, weights=w, soft_coef=0.6, label_coef=0.4)


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("temperature,dtype", [(2.0, BF16), (0.5, F32), (4.0, F32), (1.7, BF16)])
def test_temperatures_with_and_without_labels(temperature, dtype, rest):
    x, ids, values, labels, w = make(6, 5003, 24, dtype, seed=3, rest=rest, temperature=temperature)
    own = 1.0 if rest else temperature
    check(x, ids, values, temperature=temperature, teacher_temperature=own, rest=rest)
    check(x, ids, values, temperature=temperature, teacher_temperature=own, rest=rest, labels=labels, weights=w, soft_coef=1.5, label_coef=0.25)
    check(x, ids, values, temperature=temperature, teacher_temperature=own, rest=rest, labels=labels, weights=w, soft_coef=0.0, label_coef=1.0)


@pytest.mark.parametrize("rows,vocab,dtype", [(296, 2000, BF16), (30, 50257, BF16), (150, 20000, F32), (2, 300000, F32), (2, 425984, F32), (1, 851968, BF16), (700, 1001, BF16)])
def test_shapes_of_blocks_and_clusters(rows, vocab, dtype):
    x, ids, values, labels, w = make(rows, vocab, 32, dtype, seed=vocab, rest=True)
    pick = slice(0, rows) if rows <= 30 else slice(rows - 20, rows)
    labels[:: 5] = -100
    loss, sums, dx = call(x, ids, values, rest=True, labels=labels, weights=w, soft_coef=0.5, label_coef=0.5, temperature=1.3)
    want = R.distillation(x[pick], ids[pick], values[pick], rest=True, labels=labels[pick], weights=w[pick], soft=0.5, hard=0.5, temperature=1.3)
    near(loss[pick], want["token_loss"], want["token_bound"])
    near(dx[pick], want["dlogits"], want["grad_bound"] + R.half_step(dtype) * want["dlogits"].abs())
    # The totals against the losses that are checked: binary64 sums, rounded for a block and once.
    on = ((labels >= 0).double() * w.double())
    assert abs(float(sums[0]) - float((on * loss.double()).sum())) <= 8 * R.ULP * float((on * loss.double().abs()).sum())
    assert abs(float(sums[3]) - float(on.sum())) <= 8 * R.ULP * float(on.sum())
    without, s2, _ = call(x, ids, values, out=None, rest=True, labels=labels, weights=w, soft_coef=0.5, label_coef=0.5, temperature=1.3)
    assert torch.equal(loss, without) and torch.equal(sums, s2)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("offset,extra", [(1, 0), (3, 1), (5, 7), (0, 3), (8, 16)])
def test_strides_in_place_and_other_phases(dtype, offset, extra):
    more = dict(rest=True, soft_coef=0.7, label_coef=0.3)
    new = lambda: make(5, 2051, 30, dtype, seed=offset, rest=True, ld=2051 + extra, offset=offset)  # noqa: E731
    x, ids, values, labels, w = new()
    labels[0], labels[1] = 0, 2050                       # the elements beside the whole pieces
    ids[2, :6] = torch.tensor([0, 1, 2, 2048, 2049, 2050], dtype=torch.int32)
    ids[2, 6:] = -1
    wide_ids, wide = torch.full((5, 37), 7, dtype=torch.int32, device="cuda"), torch.full((5, 33), 9.0, device="cuda")
    wide_ids[:, :30], wide[:, :30] = ids, values
    _, _, apart, _ = check(x, wide_ids[:, :30], wide[:, :30], labels=labels, weights=w, **more)
    out = torch.full((5, 2060), 5.0, dtype=dtype, device="cuda")[:, 2:2053]
    check(x, ids, values, labels=labels, weights=w, out=out, **more)
    _, _, inside = call(x, ids, values, labels=labels, weights=w, in_place=True, **more)
    assert torch.equal(apart, inside)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", ["labels", "weights", "none", "one", "runs"])
def test_many_rows_of_which_some_take_part(kind, dtype):
    """Enough rows for every block to have several: they are taken in an order of their own."""
    rows = 6007
    x, ids, values, labels, w = make(rows, 501, 5, dtype, seed=20, rest=True)
    drop = torch.rand(rows, generator=gpu(21), device="cuda") < 0.4
    if kind == "labels":
        labels[drop] = -100
    elif kind == "weights":
        w[drop] = 0.0
    elif kind == "none":
        w[:] = 0.0
    elif kind == "one":
        labels[:] = -1
        labels[3000] = 7
    else:
        labels[100:4000] = 501
    off = (labels < 0) | (labels >= 501) | (w == 0)
    x[off] = math.nan
    values[off] = math.nan
    more = dict(rest=True, labels=labels, weights=w, label_coef=0.5, temperature=1.3)
    loss, sums, dx = call(x, ids, values, **more)
    on = torch.nonzero(~off)[:, 0]
    pick = on[torch.randperm(len(on), generator=gpu(22), device="cuda")[:40]]
    assert bool((loss[off] == 0).all()) and bool((dx[off] == 0).all())
    if len(pick):
        want = R.distillation(x[pick], ids[pick], values[pick], labels=labels[pick], weights=w[pick], temperature=1.3, rest=True, hard=0.5)
        near(loss[pick], want["token_loss"], want["token_bound"])
        near(dx[pick], want["dlogits"], want["grad_bound"] + R.half_step(dtype) * want["dlogits"].abs())
    part = torch.where(off, torch.zeros_like(w), w).double()
    assert abs(float(sums[0]) - float((part * loss.double()).sum())) <= 8 * R.ULP * float((part * loss.double().abs()).sum())
    assert abs(float(sums[3]) - float(part.sum())) <= 8 * R.ULP * float(part.sum())
    again = call(x, ids, values, in_place=True, **more)
    assert torch.equal(again[0], loss) and torch.equal(again[1], sums) and torch.equal(again[2], dx)


def test_inactive_rows_are_not_read():
    x, ids, values, labels, w = make(7, 3001, 9, BF16, seed=5)
    labels[1], labels[2], w[3] = -100, 3001, 0.0
    x[1:4] = math.nan
    values[1:4] = math.nan
    x[5] = -math.inf
    loss, _, dx, _ = check(x, ids, values, labels=labels, weights=w, label_coef=0.5)
    for t in (1, 2, 3, 5):
        assert float(loss[t]) == 0.0 and float(dx[t].abs().max()) == 0.0


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_masked_logits_infinities_and_nans(dtype, rest):
    x, ids, values, labels, w = make(11, 1003, 6, dtype, seed=6, rest=rest)
    low = torch.finfo(dtype).min
    every = torch.arange(1003, device="cuda")
    x[0, ids[0].long()] = -math.inf                      # the listed ones cannot happen: an infinite loss
    x[1, 3] = math.nan
    x[2, 3] = math.inf
    x[3, ids[3, 2].long()] = math.nan                    # a listed one
    x[4, ~torch.isin(every, ids[4].long())] = -math.inf  # nothing but the listed ones
    x[5, ~torch.isin(every, ids[5].long())] = low
    x[6] = low
    values[7, 2] = math.nan
    values[8, 2:] = -math.inf                            # probabilities of 0
    values[9] = -math.inf                                # nothing is listed
    ids[10] = -1
    labels[:] = ids[:, 0].long().clamp(min=0)
    check(x, ids, values, rest=rest, weights=w)
    check(x, ids, values, rest=rest, weights=w, labels=labels, label_coef=0.5, soft_coef=0.5)


@pytest.mark.parametrize("rest", [False, True])
def test_a_student_that_is_sure(rest):
    """The rest's probability far below 1 - the listed ones in binary32, and below binary32 altogether."""
    for gap in (12.0, 25.0, 60.0, 120.0, 3000.0):
        x, ids, values, labels, w = make(4, 2003, 5, F32, seed=7, rest=rest)
        x[torch.arange(4, device="cuda"), ids[:, 0].long()] = gap
        labels[0] = ids[0, 0]
        check(x, ids, values, rest=rest, weights=w, labels=labels, label_coef=0.5)


@pytest.mark.parametrize("temperature,k", [(4.0, 3), (2.0, 40), (3.3, 1), (1.0, 128)])
@pytest.mark.parametrize("rest", [False, True])
def test_small_losses_keep_their_digits(temperature, k, rest):
    """Flat distributions, of which the list is a small part: the loss is made of logarithms that nearly cancel.  They are
    off by what the student's sum is, 2 half steps, and by the temperature's rounding times an exponent of about 10; the
    terms' d^2 / 2 with d of about 0.7 / temperature by that over d / 2."""
    x, ids, values, _, _ = make(40, 20011, k, BF16, seed=30, rest=rest, temperature=temperature)
    more = dict(rest=rest, temperature=temperature, teacher_temperature=1.0 if rest else temperature)
    loss, _, _, want = check(x, ids, values, **more)
    off = float((loss.double() - want["token_loss"]).norm() / want["token_loss"].norm())
    assert off <= R.ULP * (2 + 10) * temperature / 0.7 * 2, off


def test_teacher_and_student_alike():
    """Near 0 the loss keeps its digits: its terms are of one sign."""
    from paper_2512_09685_b200 import binding as B
    x, _, _, _, _ = make(6, 5003, 40, F32, seed=8)
    ids, top = torch.empty((6, 40), dtype=torch.int32, device="cuda"), torch.empty((6, 40), device="cuda")
    B.star_token_alternatives(x, ids, top)
    y = x + 1e-3 * torch.randn(x.shape, generator=gpu(9), device="cuda")
    loss, _, _, want = check(y, ids, top, rest=True)
    # Terms q (exp(d) - 1 - d) of log ratios d about 1e-3, each good to a few 1e-6 / 1e-3.
    assert float(((loss.double() - want["token_loss"]).abs() / want["token_loss"]).max()) <= 2e-2
    same, _, dx = call(x, ids, top, rest=True)
    assert float(same.abs().max()) <= 64 * R.ULP and float(dx.abs().max()) <= 64 * R.ULP


@pytest.mark.parametrize("rest", [False, True])
def test_the_same_id_twice_and_ids_out_of_range(rest):
    x, ids, values, labels, w = make(4, 2001, 7, F32, seed=10, rest=rest)
    ids[0] = torch.tensor([5, 5, 5, 9, -1, 2001, 5], dtype=torch.int32)
    ids[1] = torch.tensor([0, 2000, 0, 2000, 7, 7, 7], dtype=torch.int32)
    ids[2] = -1
    values[0:2] = math.log(0.1) if rest else 1.0
    labels[0], labels[1] = 5, 2000
    check(x, ids, values, rest=rest, weights=w)
    check(x, ids, values, rest=rest, weights=w, labels=labels, label_coef=0.3, temperature=2.0)


def test_probabilities_of_more_than_one():
    x, ids, values, _, w = make(3, 2001, 4, F32, seed=11, rest=True)
    values[:] = math.log(0.4)
    check(x, ids, values, rest=True, weights=w)


def test_no_teacher_is_cross_entropy():
    x, _, _, labels, w = make(5, 2001, 1, F32, seed=12)
    ids, values = torch.empty((5, 0), dtype=torch.int32, device="cuda"), torch.empty((5, 0), device="cuda")
    check(x, ids, values, labels=labels, weights=w, soft_coef=0.0, label_coef=1.0)
    check(x, ids, values, labels=labels, weights=w, soft_coef=1.0, label_coef=1.0, rest=True)


def test_nothing_to_do():
    ids, values = torch.empty((0, 3), dtype=torch.int32, device="cuda"), torch.empty((0, 3), device="cuda")
    _, sums, _ = call(torch.empty((0, 100), device="cuda"), ids, values)
    assert sums.tolist() == [0.0] * 4
    ids, values = torch.zeros((2, 3), dtype=torch.int32, device="cuda"), torch.zeros((2, 3), device="cuda")
    loss, sums, _ = call(torch.empty((2, 0), device="cuda"), ids, values)
    assert loss.tolist() == [0.0] * 2 and sums.tolist() == [0.0] * 4


def test_the_same_call_gives_the_same_bits():
    x, ids, values, labels, w = make(700, 5003, 64, BF16, seed=13, rest=True)
    a = call(x, ids, values, rest=True, labels=labels, weights=w, label_coef=0.5)
    b = call(x, ids, values, rest=True, labels=labels, weights=w, label_coef=0.5)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("rest", [False, True])
def test_gradient_against_differences(rest):
    x, ids, values, labels, w = make(3, 501, 8, F32, seed=14, rest=rest, temperature=1.5)
    more = dict(rest=rest, labels=labels, weights=w, label_coef=0.4, soft_coef=0.8, temperature=1.5)
    _, _, dx = call(x, ids, values, **more)
    step = 2.0 ** -6
    for seed in range(3):
        v = torch.randn(x.shape, generator=gpu(seed), device="cuda")
        v = v / v.norm()
        up, down = (float(call(x + s * step * v, ids, values, out=None, **more)[1][0]) for s in (1, -1))
        # Third derivatives of order 1 along a direction of length 1; sums of about 20, off by 20 half steps.
        assert abs((up - down) / (2 * step) - float((dx.double() * v.double()).sum())) <= step ** 2 + 20 * R.ULP * 20 / step


def test_a_wait_that_runs_out():
    from paper_2512_09685_b200 import binding as B
    x, ids, values, _, _ = make(700, 5003, 8, BF16, seed=15)
    few, few_ids, few_values, _, _ = make(3, 200000, 8, BF16, seed=15)
    B.star_check_waits()
    B.star_set_wait_attempts(0)
    try:
        for a in ((x, ids, values), (few, few_ids, few_values)):
            loss, sums = torch.zeros(a[0].shape[0], device="cuda"), torch.zeros(4, device="cuda")
            ws = torch.empty(B.star_loss_workspace_bytes(a[0].shape[0]), dtype=torch.uint8, device="cuda")
            B.star_distillation_loss(*a, loss, sums, ws, dlogits=torch.empty_like(a[0]))
            with pytest.raises(B.StarError) as e:
                B.star_check_waits()
            assert e.value.status == B.STAR_ERR_TIMEOUT
            assert bool(torch.isnan(sums).all())
    finally:
        B.star_set_wait_attempts()
    check(x[:20], ids[:20], values[:20])
