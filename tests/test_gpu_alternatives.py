"""Log-probabilities with entropy and top alternatives, and their backward pass,
against the formulas in binary64.  Bounds count half steps of binary32 (and the one
rounding to bf16); ids have to be equal."""
import math

import pytest
import torch

from . import distillation_reference as R

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def gpu(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def make(rows, vocab, dtype, seed=0, spread=2.0, ld=None, offset=0):
    g = gpu(seed)
    ld = ld or vocab
    store = torch.full((offset + rows * ld + 64,), 7.0, dtype=dtype, device="cuda")
    x = store[offset:offset + rows * ld].view(rows, ld)[:, :vocab]
    x.copy_(torch.randn((rows, vocab), generator=g, device="cuda") * spread)
    return x


def call(x, k, labels=None, temperature=1.0, ld_top=None):
    from paper_2512_09685_b200 import binding as B
    rows = x.shape[0]
    wide = max(ld_top or k, 1)
    ids = torch.full((rows, wide), -77, dtype=torch.int32, device="cuda")
    top = torch.full((rows, wide), 77.0, device="cuda")
    lse, entropy = torch.full((rows,), 77.0, device="cuda"), torch.full((rows,), 77.0, device="cuda")
    logp = None if labels is None else torch.full((rows,), 77.0, device="cuda")
    B.star_token_alternatives(x, ids[:, :k] if k else None, top[:, :k] if k else None, labels=labels, logp=logp, lse=lse, entropy=entropy,
                              temperature=temperature)
    torch.cuda.synchronize()
    assert bool((ids[:, k:] == -77).all()) and bool((top[:, k:] == 77.0).all())
    return {"ids": ids[:, :k], "top": top[:, :k], "lse": lse, "entropy": entropy, "logp": logp}


def close(got, want, bound):
    got, want = got.double(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    far = torch.isinf(want)
    assert torch.equal(got[far], want[far])
    fine = torch.isfinite(want)
    off = (got - want).abs()
    assert bool((off[fine] <= bound.expand_as(off)[fine]).all()), float((off[fine] / bound.expand_as(off)[fine]).max())


def check(got, want, k):
    assert torch.equal(got["ids"].long(), want["ids"])
    fine = torch.where(want["active"][:, None] & torch.isfinite(want["lse"])[:, None], want["every"], torch.zeros_like(want["every"]))
    close(got["top"], want["top"], R.log_bound(torch.where(torch.isfinite(want["top"]), want["top"], torch.zeros_like(want["top"])), fine))
    finite = lambda v: torch.where(torch.isfinite(v), v, torch.zeros_like(v))  # noqa: E731
    one = R.log_bound(torch.zeros_like(want["lse"])[:, None], fine)[:, 0]
    close(got["lse"], want["lse"], one + 8 * R.ULP * finite(want["lse"]).abs())
    close(got["entropy"], want["entropy"], one * (1 + finite(want["entropy"])))
    if got["logp"] is not None:
        close(got["logp"], want["logp"], one + 8 * R.ULP * finite(want["logp"]).abs())


SIZES = [(1, 1, 1, F32), (3, 5, 8, BF16), (1, 50257, 20, BF16), (5, 50257, 64, BF16), (7, 32001, 8, F32), (4, 2000, 128, BF16), (4, 1000, 128, F32),
         (6, 1024, 128, BF16), (130, 129, 3, BF16), (2, 131072, 128, F32), (300, 257, 17, F32), (2, 200000, 100, BF16), (9, 4097, 1, BF16), (3, 64, 0, F32),
         (700, 3001, 33, BF16)]


@pytest.mark.parametrize("rows,vocab,k,dtype", SIZES)
def test_sizes(rows, vocab, k, dtype):
    x = make(rows, vocab, dtype, seed=rows + vocab)
    labels = torch.randint(0, vocab, (rows,), generator=gpu(1), device="cuda")
    check(call(x, k, labels), R.alternatives(x, k, labels), k)
    check(call(x, k), R.alternatives(x, k), k)


@pytest.mark.parametrize("temperature", [0.25, 2.0, 7.5])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_temperatures(temperature, dtype):
    x = make(5, 5003, dtype, seed=3)
    labels = torch.randint(0, 5003, (5,), generator=gpu(1), device="cuda")
    check(call(x, 10, labels, temperature), R.alternatives(x, 10, labels, temperature), 10)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("offset,extra", [(1, 0), (3, 1), (5, 7), (8, 16), (0, 3)])
def test_strides_and_phases(dtype, offset, extra):
    x = make(6, 2051, dtype, seed=offset, ld=2051 + extra, offset=offset)
    check(call(x, 30, ld_top=37), R.alternatives(x, 30), 30)


def test_masked_rows_are_not_read():
    x = make(8, 3000, BF16, seed=5)
    x[2] = math.nan
    labels = torch.tensor([0, 2999, -100, 3000, 17, -1, 5, 1 << 40], device="cuda")
    got = call(x, 5, labels)
    check(got, R.alternatives(x, 5, labels), 5)
    for t in (2, 3, 5, 7):
        assert got["ids"][t].tolist() == [-1] * 5 and float(got["lse"][t]) == -math.inf and float(got["logp"][t]) == 0.0 and float(got["entropy"][t]) == 0.0


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_infinities_and_nans(dtype):
    x = make(9, 4099, dtype, seed=6)
    x[0] = -math.inf
    x[1, 7] = math.nan
    x[2, 4098] = math.inf
    x[3] = -math.inf
    x[3, 4000] = 1.5                                     # one possible token
    x[4] = -math.inf
    x[4, 100:110] = torch.arange(10, device="cuda").to(dtype)
    x[5] = torch.finfo(dtype).min                        # a mask of the lowest value, all of it
    x[6] = torch.finfo(dtype).min
    x[6, 11] = 3.0
    x[7, ::2] = -math.inf
    x[8] = -0.0
    x[8, 1::2] = 0.0                                     # both zeros are one value
    got = call(x, 20)
    check(got, R.alternatives(x, 20), 20)
    assert got["ids"][8].tolist() == list(range(20))
    assert got["ids"][3].tolist() == [4000] + [-1] * 19 and float(got["top"][3, 0]) == 0.0 and float(got["entropy"][3]) == 0.0
    assert got["ids"][5].tolist() == list(range(20))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("k", [1, 20, 128])
def test_rows_with_many_candidates(dtype, k):
    """Equal logits, two values, large ones side by side, sorted rows: what leaves more than the usual number to choose from."""
    V = 20011
    g = gpu(8)
    x = torch.zeros((9, V), device="cuda")
    x[1] = torch.randint(0, 2, (V,), generator=g, device="cuda").float()
    x[2] = torch.randint(0, 30, (V,), generator=g, device="cuda").float()
    x[3, 1000:3000] = 5 + torch.randn(2000, generator=g, device="cuda")
    x[4] = torch.arange(V, device="cuda") / V
    x[5] = -torch.arange(V, device="cuda") / V
    x[6, :] = torch.randn(V, generator=g, device="cuda")
    x[6, 8::2048] = 9.0                                  # one thread's elements
    x[6, 9::2048] = 9.0
    x[7] = -1e30
    x[7, -300:] = 1.0                                    # the row's end, its last piece among it
    x[8] = torch.randn(V, generator=g, device="cuda") * 1e-30
    x = x.to(dtype)
    check(call(x, k), R.alternatives(x, k), k)


def test_the_same_call_gives_the_same_bits():
    x = make(64, 50257, BF16, seed=9)
    a, b = call(x, 64), call(x, 64)
    assert all(torch.equal(a[n], b[n]) for n in ("ids", "top", "lse", "entropy"))


def test_nothing_to_do():
    from paper_2512_09685_b200 import binding as B
    x = torch.empty((0, 100), device="cuda")
    B.star_token_alternatives(x, torch.empty((0, 4), dtype=torch.int32, device="cuda"), torch.empty((0, 4), device="cuda"))
    got = call(torch.empty((3, 0), device="cuda"), 2)
    assert got["ids"].tolist() == [[-1, -1]] * 3 and got["lse"].tolist() == [-math.inf] * 3 and got["entropy"].tolist() == [0.0] * 3


def test_more_than_2_31_elements():
    """Rows whose offsets pass 32 bits: the last ones."""
    rows, vocab = 43000, 50257
    x = torch.zeros((rows, vocab), dtype=BF16, device="cuda")
    x[-3:] = torch.randn((3, vocab), generator=gpu(2), device="cuda").to(BF16)
    labels = torch.full((rows,), -100, dtype=torch.int64, device="cuda")
    labels[-3:] = 5
    got = call(x, 10, labels)
    want = R.alternatives(x[-3:], 10, labels[-3:])
    check({n: v[-3:] for n, v in got.items()}, want, 10)
    dx = torch.full_like(x, 3.0)
    from paper_2512_09685_b200 import binding as B
    d = torch.ones(rows, device="cuda")
    B.star_token_alternatives_backward(dx, x, got["lse"], labels=labels, d_logp=d)
    g, bound = R.alternatives_backward(x[-3:], got["lse"][-3:], labels[-3:], d[-3:])
    assert bool(((dx[-3:].double() - g).abs() <= bound + R.half_step(BF16) * g.abs()).all())
    assert float(dx[:-3].abs().max()) == 0.0


# ---------------------------------------------------------------------------
# Backward
# ---------------------------------------------------------------------------
def backward(x, k, labels=None, temperature=1.0, names=("d_logp", "d_entropy", "d_top"), seed=0, in_place=False, out=None, ids=None):
    from paper_2512_09685_b200 import binding as B
    g = gpu(seed + 100)
    rows = x.shape[0]
    fwd = call(x, k, labels, temperature)
    a = {"d_logp": torch.randn(rows, generator=g, device="cuda") if labels is not None and "d_logp" in names else None,
         "d_entropy": torch.randn(rows, generator=g, device="cuda") if "d_entropy" in names else None}
    top_ids = d_top = None
    if k and "d_top" in names:
        top_ids = fwd["ids"].contiguous() if ids is None else ids
        d_top = torch.randn(top_ids.shape, generator=g, device="cuda")
    want, bound = R.alternatives_backward(x, fwd["lse"], labels, a["d_logp"], fwd["entropy"], a["d_entropy"], top_ids, d_top, temperature)
    dx = x if in_place else torch.full_like(x, 5.0) if out is None else out
    B.star_token_alternatives_backward(dx, x, fwd["lse"], labels=labels, d_logp=a["d_logp"], entropy=fwd["entropy"], d_entropy=a["d_entropy"],
                                       top_ids=top_ids, d_top_logp=d_top, temperature=temperature)
    torch.cuda.synchronize()
    bad = torch.isnan(want)
    assert torch.equal(torch.isnan(dx), bad)
    off = (dx.double() - want).abs() - bound - R.half_step(x.dtype) * want.abs()
    assert bool((off[~bad] <= 0).all()), float(off[~bad].max())
    return dx, want


@pytest.mark.parametrize("rows,vocab,k,dtype", [s for s in SIZES if s[1] < 140000])
def test_backward_sizes(rows, vocab, k, dtype):
    x = make(rows, vocab, dtype, seed=rows + vocab)
    labels = torch.randint(0, vocab, (rows,), generator=gpu(1), device="cuda")
    backward(x, k, labels)
    backward(x, k, None, 2.5)


@pytest.mark.parametrize("names", [("d_logp",), ("d_entropy",), ("d_top",), ("d_logp", "d_entropy"), ()])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_backward_of_some_results(names, dtype):
    x = make(11, 2003, dtype, seed=4)
    labels = torch.randint(0, 2003, (11,), generator=gpu(1), device="cuda")
    labels[3] = -100
    dx, _ = backward(x, 6, labels, names=names)
    assert float(dx[3].abs().max()) == 0.0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("offset,extra", [(1, 0), (3, 1), (0, 3), (8, 16)])
def test_backward_strides_in_place_and_other_phases(dtype, offset, extra):
    labels = torch.randint(0, 2051, (6,), generator=gpu(1), device="cuda")
    make_x = lambda: make(6, 2051, dtype, seed=offset, ld=2051 + extra, offset=offset)  # noqa: E731
    apart, _ = backward(make_x(), 30, labels)
    inside, _ = backward(make_x(), 30, labels, in_place=True)
    assert torch.equal(apart, inside)
    out = torch.full((6, 2060), 5.0, dtype=dtype, device="cuda")[:, 2:2053]
    backward(make_x(), 30, labels, out=out)


def test_backward_with_the_same_id_twice_and_ids_out_of_range():
    V = 3001
    x = make(4, V, F32, seed=12)
    labels = torch.tensor([10, 20, 30, 40], device="cuda")
    ids = torch.tensor([[10, 10, 10, -1, V, 7], [1, 2, 1, 2, 1, 2], [0, V - 1, V - 1, 0, 30, 30], [-1] * 6], dtype=torch.int32, device="cuda")
    backward(x, 6, labels, ids=ids)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_backward_of_masked_logits(dtype):
    x = make(6, 1003, dtype, seed=13)
    x[0] = -math.inf
    x[1, 5] = math.nan
    x[2, ::2] = -math.inf
    x[3] = torch.finfo(dtype).min
    x[3, 9] = 1.0
    x[4, 3:] = -math.inf
    labels = torch.tensor([1, 1, 2, 9, 1, 0], device="cuda")
    dx, _ = backward(x, 8, labels)
    assert float(dx[0].abs().max()) == 0.0 and bool(torch.isnan(dx[1]).all())


def test_backward_against_differences():
    """The results' change along a direction; binary32 results are good to 1e-6 here, the step is 2^-6."""
    x = make(3, 501, F32, seed=14)
    labels = torch.tensor([3, 400, 77], device="cuda")
    g = gpu(15)
    d_logp, d_entropy = torch.randn(3, generator=g, device="cuda"), torch.randn(3, generator=g, device="cuda")
    from paper_2512_09685_b200 import binding as B
    base = call(x, 4, labels)
    d_top = torch.randn((3, 4), generator=g, device="cuda")
    dx = torch.empty_like(x)
    B.star_token_alternatives_backward(dx, x, base["lse"], labels=labels, d_logp=d_logp, entropy=base["entropy"], d_entropy=d_entropy,
                                       top_ids=base["ids"].contiguous(), d_top_logp=d_top)

    def value(y):
        r = call(y, 4, labels)
        assert torch.equal(r["ids"], base["ids"])
        return float((r["logp"] * d_logp + r["entropy"] * d_entropy).double().sum() + (r["top"] * d_top).double().sum())

    step = 2.0 ** -6
    for seed in range(3):
        v = torch.randn(x.shape, generator=gpu(seed), device="cuda")
        v = v / v.norm()
        slope = (value(x + step * v) - value(x - step * v)) / (2 * step)
        # Third derivatives of order 1, of a direction of length 1: step^2; results off by 20 half steps of about 8.
        assert abs(slope - float((dx.double() * v.double()).sum())) <= step ** 2 + 20 * 2.0 ** -24 * 8 / step
