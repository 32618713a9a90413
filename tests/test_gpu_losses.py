"""The losses over the vocabulary on the GPU against their formulas in binary64.

Tolerances (2-norm over 2-norm unless said otherwise), derived before the first
run.  u = 2^-24 is binary32's rounding unit.
  logp: the sum of exponentials is off by at most ~2 ulp per term of ex2 plus
      the additions' (pairwise over >= 32 lanes, a few hundred terms each): below
      64 u relative, i.e. 4e-6 absolute on logp and lse in the worst case; the
      difference to the label's logit and the logarithm add a few u of the result.
      Bound: 4e-6 absolute + 4e-7 relative.
  dlogits fp32: p is off by the sum's error (4e-6) and by u |x - m| log2(e) of the
      exponent's product, |x - m| < 60 here: 8e-6; the factor by expf of a value
      that is off by 4e-6.  Bound 2e-5.
  dlogits bf16: one rounding to 8 significant bits, at most 2^-8 = 3.9e-3 each: bound 4e-3.
  loss terms: exp of logp's error: bound 1e-5 of the largest term involved.
"""
import itertools
import math

import pytest
import torch

from tests import worker_step_reference as R

pytestmark = pytest.mark.gpu

LOGP_ABS, LOGP_REL = 4e-6, 4e-7
GRAD = {torch.float32: 2e-5, torch.bfloat16: 4e-3}
LOSS = 1e-5


@pytest.fixture(scope="module")
def B():
    from paper_2512_09685_b200 import binding
    return binding


def make(T, V, dtype, seed, std=2.0, offset=0, pad=0, masked=0.25):
    """Logits with a row stride of V + pad that start `offset` elements into their storage."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    ld = V + pad
    store = torch.full((offset + T * ld + 64,), 1e30, device="cuda").to(dtype)
    x = store[offset: offset + T * ld].view(T, ld)[:, :V]
    x.copy_(torch.randn((T, V), generator=g, device="cuda") * std)
    labels = torch.randint(0, V, (T,), generator=g, device="cuda")
    drop = torch.rand(T, generator=g, device="cuda") < masked
    labels[drop] = torch.where(torch.rand(int(drop.sum()), generator=g, device="cuda") < 0.5, -100, V + 5)
    return x, labels, g


def close(got, want, absolute=LOGP_ABS, relative=LOGP_REL):
    got, want = got.double(), want.double()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    return bool((same | ((got - want).abs() <= absolute + relative * want.abs())).all())


def policy_call(B, x, labels, A, dlogits="new", **kw):
    T, V = x.shape
    out = {"logp": torch.full((T,), 7.0, device="cuda"), "token_loss": torch.full((T,), 7.0, device="cuda"),
           "sums": torch.full((4,), 7.0, device="cuda")}
    ws = torch.full((B.star_loss_workspace_bytes(T),), 255, dtype=torch.uint8, device="cuda")
    d = None
    if dlogits == "new":
        d = torch.full((T, V), 7.0, device="cuda").to(x.dtype)
    elif dlogits is not None:
        d = dlogits
    B.star_policy_loss(x, labels, A, out["logp"], out["token_loss"], out["sums"], ws, dlogits=d, **kw)
    torch.cuda.synchronize()
    return {**out, "dlogits": d}


# lengths around the widths of loads, warps, blocks and of one block's share of a row
VOCABS = [1, 2, 7, 8, 9, 31, 33, 127, 255, 1000, 1025, 4096, 8191, 32001, 50257]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", VOCABS + [120_011, 300_007])
def test_logprobs_over_vocabulary_sizes(B, V, dtype):
    for T in (1, 5):
        x, labels, _ = make(T, V, dtype, seed=V + T, masked=0.2)
        lp, lse = torch.full((T,), 7.0, device="cuda"), torch.full((T,), 7.0, device="cuda")
        B.star_token_logprobs(x, labels, lp, lse, temperature=0.7)
        torch.cuda.synchronize()
        want, want_lse, _, _ = R.rows(x, labels, None, 0.7)
        assert close(lp, want) and close(lse, want_lse)
        only = torch.full((T,), 7.0, device="cuda")
        B.star_token_logprobs(x, labels, only, temperature=0.7)
        assert torch.equal(only, lp)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", VOCABS)
def test_policy_loss_over_vocabulary_sizes(B, V, dtype):
    for T, (old, ref) in zip((1, 3, 40, 41), itertools.product((True, False), (True, False))):
        x, labels, g = make(T, V, dtype, seed=7 * V + T)
        lp = R.rows(x, labels)[0].float()
        A = torch.randn(T, generator=g, device="cuda")
        kw = dict(weights=torch.rand(T, generator=g, device="cuda") * (torch.rand(T, generator=g, device="cuda") < 0.9),
                  kl_coef=0.3 if ref else 0.0, clip_low=0.1, clip_high=0.3)
        shift = 0.4 * torch.randn(T, generator=g, device="cuda")
        for edge in (math.log(0.9), math.log(1.3)):       # which side of an edge rounding puts a ratio on is not tested
            shift = torch.where((shift - edge).abs() < 1e-3, shift + 4e-3, shift)
        old_lp = lp - shift if old else None
        ref_lp = lp + 0.5 * torch.randn(T, generator=g, device="cuda") if ref else None
        got = policy_call(B, x, labels, A, old_logp=old_lp, ref_logp=ref_lp, **kw)
        want = R.policy(x, labels, A, old=old_lp, ref=ref_lp, **kw)
        assert close(got["logp"], want["logp"])
        size = float((want["token_loss"].abs() + A.abs()).max())
        assert close(got["token_loss"], want["token_loss"], absolute=LOSS * max(size, 1.0))
        assert close(got["sums"], want["sums"], absolute=LOSS * T * max(size, 1.0))
        assert R.rel(got["dlogits"], want["dlogits"]) <= GRAD[dtype] or float(want["dlogits"].abs().max()) < 1e-6
        assert torch.equal(got["dlogits"][~want["active"]], torch.zeros_like(got["dlogits"][~want["active"]]))
        alone = policy_call(B, x, labels, A, dlogits=None, old_logp=old_lp, ref_logp=ref_lp, **kw)
        for name in ("logp", "token_loss", "sums"):
            assert torch.equal(alone[name], got[name]), name


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset,pad,out_offset,out_pad", [(0, 0, 0, 3), (1, 0, 1, 0), (1, 7, 5, 0), (3, 5, 0, 0), (0, 8, 0, 16),
                                                          (2, 6, 4, 1)])
@pytest.mark.parametrize("V", [5, 40, 1003, 4096, 33000])
def test_strides_and_alignments(B, V, offset, pad, out_offset, out_pad, dtype):
    T = 6
    x, labels, g = make(T, V, dtype, seed=V + offset, offset=offset, pad=pad)
    A = torch.randn(T, generator=g, device="cuda")
    ld = V + out_pad
    store = torch.full((out_offset + T * ld + 64,), 3.0, device="cuda").to(dtype)
    d = store[out_offset: out_offset + T * ld].view(T, ld)[:, :V]
    got = policy_call(B, x, labels, A, dlogits=d)
    want = R.policy(x, labels, A)
    assert close(got["logp"], want["logp"]) and R.rel(d, want["dlogits"]) <= GRAD[dtype]
    # nothing outside the matrix was written
    keep = torch.full_like(store, 3.0)
    keep[out_offset: out_offset + T * ld].view(T, ld)[:, :V] = d
    assert torch.equal(store.float(), keep.float())
    # and in place
    kept = x.clone()
    before = policy_call(B, x, labels, A)
    policy_call(B, x, labels, A, dlogits=x)
    assert torch.equal(x, before["dlogits"]) and not torch.equal(x, kept)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V", [(300, 1024), (1000, 2050), (700, 8192), (333, 50257)])
def test_many_rows(B, T, V, dtype):
    x, labels, g = make(T, V, dtype, seed=T, masked=0.4)
    A = torch.randn(T, generator=g, device="cuda")
    got, want = policy_call(B, x, labels, A), R.policy(x, labels, A)
    assert close(got["logp"], want["logp"]) and R.rel(got["dlogits"], want["dlogits"]) <= GRAD[dtype]
    again = policy_call(B, x, labels, A)
    for name in got:
        assert torch.equal(got[name], again[name]), name          # the same bits every time


def test_masked_and_special_logits(B):
    V = 1000
    for dtype in (torch.float32, torch.bfloat16):
        lowest = torch.finfo(dtype).min
        x, labels, g = make(12, V, dtype, seed=5, masked=0.0)
        A = torch.randn(12, generator=g, device="cuda")
        x[0] = -math.inf                                  # nothing left: inactive
        x[1, 10:] = -math.inf                             # few left, the label among them
        labels[1] = 3
        x[2, 10:] = lowest
        labels[2] = 9
        x[3] = lowest                                     # all at the lowest value: uniform
        x[4] = math.nan                                   # masked by its label: not read
        labels[4] = -100
        x[5] = math.inf
        labels[5] = V
        x[6, 500] = math.nan                              # active: NaN in its own row
        x[8, 7] = math.inf
        x[9, 0] = 3e38 if dtype == torch.float32 else 3e38
        labels[9] = 0
        x[10, :] = -math.inf
        x[10, 17] = -5.0
        labels[10] = 17                                   # the only possible token: probability one
        got, want = policy_call(B, x, labels, A), R.policy(x, labels, A)
        assert close(got["logp"], want["logp"])
        for t in range(12):
            w, h = want["dlogits"][t], got["dlogits"][t]
            assert bool(torch.isnan(w).any()) == bool(torch.isnan(h).any()), t
            if not bool(torch.isnan(w).any()):
                assert R.rel(h, w) <= GRAD[dtype] or float(w.abs().max()) < 1e-6, t
        assert bool(torch.isnan(got["dlogits"][6]).all()) and bool(torch.isnan(got["dlogits"][8]).all())
        assert bool((got["dlogits"][[0, 4, 5]] == 0).all()) and got["logp"][0] == 0
        assert got["logp"][10] == 0 and bool((got["dlogits"][10] == 0).all())
        assert bool(torch.isnan(got["sums"][0]))
        lse = torch.empty(12, device="cuda")
        B.star_token_logprobs(x, labels, got["logp"], lse)
        assert close(lse[[1, 2, 7, 10, 11]], R.rows(x, labels)[1][[1, 2, 7, 10, 11]])
        # a label that its own mask forbids: probability zero, logp -inf, gradient 0 for a ratio of 0 that is not clipped
        x[7, int(labels[7])] = -math.inf
        old = torch.zeros(12, device="cuda")
        A[7] = 1.0
        got = policy_call(B, x, labels, A, old_logp=old)
        assert got["logp"][7] == -math.inf and bool((got["dlogits"][7] == 0).all())


def test_weights_decide_what_is_read(B):
    x, labels, g = make(9, 500, torch.bfloat16, seed=3, masked=0.0)
    A = torch.randn(9, generator=g, device="cuda")
    w = torch.ones(9, device="cuda")
    w[2], w[5] = 0.0, -0.0
    x[2] = math.nan
    x[5] = math.nan
    got = policy_call(B, x, labels, A, weights=w)
    assert bool(torch.isfinite(got["dlogits"].float()).all()) and bool((got["logp"][[2, 5]] == 0).all())


def test_policy_gradient_against_differences(B):
    """Central differences of the forward pass's own loss.  Step h = 2^-6: the
    loss (sum of 4 terms of order 1, each off by 1e-6) contributes 4e-6 / 2h =
    1.3e-4, the third derivative h^2 / 6 of order 1 another 4e-5."""
    T, V, h = 4, 37, 2.0 ** -6
    x, labels, g = make(T, V, torch.float32, seed=11, masked=0.0)
    A = torch.randn(T, generator=g, device="cuda")
    lp = R.rows(x, labels, None, 1.5)[0].float()
    kw = dict(old_logp=lp - 0.05, ref_logp=lp + 0.3, kl_coef=0.4, temperature=1.5)
    d = policy_call(B, x, labels, A, **kw)["dlogits"]
    for t, j in [(0, 0), (1, int(labels[1])), (2, 36), (3, 5), (3, int(labels[3]))]:
        up, down = x.clone(), x.clone()
        up[t, j] += h
        down[t, j] -= h
        slope = (float(policy_call(B, up, labels, A, dlogits=None, **kw)["sums"][0])
                 - float(policy_call(B, down, labels, A, dlogits=None, **kw)["sums"][0])) / (2 * h)
        assert abs(slope - float(d[t, j])) <= 2e-4, (t, j)


def preference_call(B, x, labels, offsets, dlogits="new", **kw):
    T, V = x.shape
    P = (len(offsets) - 1) // 2
    out = {"seq_logp": torch.full((2 * P,), 7.0, device="cuda"), "pair_loss": torch.full((P,), 7.0, device="cuda"),
           "margin": torch.full((P,), 7.0, device="cuda"), "loss": torch.full((1,), 7.0, device="cuda")}
    ws = torch.full((B.star_loss_workspace_bytes(T, 2 * P),), 255, dtype=torch.uint8, device="cuda")
    d = torch.full((T, V), 7.0, device="cuda").to(x.dtype) if isinstance(dlogits, str) else dlogits
    B.star_preference_loss(x, labels, torch.tensor(offsets, dtype=torch.int32, device="cuda"), out["seq_logp"],
                           out["pair_loss"], out["margin"], out["loss"], ws, dlogits=d, **kw)
    torch.cuda.synchronize()
    return {**out, "dlogits": d}


PAIRS = [
    [0, 3, 7],                                   # one pair
    [0, 1, 2, 2, 2, 9, 30],                      # single tokens, an empty pair, ragged
    [2, 5, 5, 20, 31, 40, 40, 41, 70],           # rows before the first and after the last sequence belong to none
    [0, 0, 0],                                   # nothing at all
]


def check_preference(got, want, dtype, beta, tokens):
    assert close(got["seq_logp"], want["seq_logp"], absolute=LOGP_ABS * tokens)
    assert close(got["margin"], want["margin"], absolute=2 * abs(beta) * LOGP_ABS * tokens)
    assert close(got["pair_loss"], want["pair_loss"], absolute=2 * abs(beta) * LOGP_ABS * tokens, relative=1e-6)
    assert close(got["loss"], want["loss"], absolute=2 * abs(beta) * LOGP_ABS * tokens * max(1, len(want["margin"])), relative=1e-6)
    # a factor's relative error is that of a sigmoid: the margin's absolute error
    bound = GRAD[dtype] + 2 * abs(beta) * LOGP_ABS * tokens
    assert R.rel(got["dlogits"], want["dlogits"]) <= bound or float(want["dlogits"].abs().max() if want["dlogits"].numel() else 0) < 1e-6


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offsets", PAIRS)
@pytest.mark.parametrize("V", [1, 9, 130, 1025, 9000])
def test_preference_loss(B, V, offsets, dtype):
    T = 75 if offsets[-1] > 40 else max(offsets[-1], 1)
    x, labels, g = make(T, V, dtype, seed=V + T)
    ref = 3 * torch.randn(len(offsets) - 1, generator=g, device="cuda")
    for kw in (dict(beta=0.1), dict(beta=0.7, label_smoothing=0.2, average=True, loss_scale=0.25, ref_logp=ref),
               dict(beta=2.0, label_smoothing=1.0, ref_logp=ref, temperature=1.3)):
        got = preference_call(B, x, labels, offsets, **kw)
        want = R.preference(x, labels, offsets, ref=kw.get("ref_logp"), beta=kw["beta"], smoothing=kw.get("label_smoothing", 0.0),
                            average=kw.get("average", False), scale=kw.get("loss_scale", 1.0), temperature=kw.get("temperature", 1.0))
        check_preference(got, want, dtype, kw["beta"], T)
        alone = preference_call(B, x, labels, offsets, dlogits=None, **kw)
        for name in ("seq_logp", "pair_loss", "margin", "loss"):
            assert torch.equal(alone[name], got[name]), name
    inplace = x.clone()
    preference_call(B, inplace, labels, offsets, dlogits=inplace, **kw)
    assert torch.equal(inplace, got["dlogits"])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_preference_loss_with_many_rows(B, dtype):
    offsets = [0, 200, 301, 302, 900, 1000, 1300, 1600, 1999]
    x, labels, g = make(2000, 6001, dtype, seed=8, masked=0.5)
    got = preference_call(B, x, labels, offsets, beta=0.01)
    want = R.preference(x, labels, offsets, beta=0.01)
    check_preference(got, want, dtype, 0.01, 600)
    again = preference_call(B, x, labels, offsets, beta=0.01)
    for name in got:
        assert torch.equal(got[name], again[name]), name


def test_preference_loss_at_extreme_margins(B):
    x, labels, _ = make(4, 16, torch.float32, seed=2, masked=0.0)
    for side in (1.0, -1.0):
        ref = torch.tensor([side * 4000.0, 0.0], device="cuda")
        got = preference_call(B, x, labels, [0, 2, 4], beta=1.0, ref_logp=ref)
        want = R.preference(x, labels, [0, 2, 4], beta=1.0, ref=ref)
        check_preference(got, want, torch.float32, 1.0, 4)
        assert bool(torch.isfinite(got["dlogits"]).all())


def test_offsets_outside_the_rows_stay_inside_the_buffers(B):
    x, labels, _ = make(20, 50, torch.float32, seed=2)
    for offsets in ([-5, 4, 100], [0, 2 ** 31 - 1, 20], [15, 3, -1]):
        got = preference_call(B, x, labels, offsets)
        assert bool(torch.isfinite(got["dlogits"]).all())


def test_preference_gradient_against_differences(B):
    """As for the policy loss: the loss is off by 2 beta * 20 tokens * 1e-6, over
    2h = 2^-5: 3e-4 of beta = 0.25's slope scale."""
    h, offsets = 2.0 ** -6, [0, 4, 9, 12, 20]
    x, labels, g = make(20, 23, torch.float32, seed=21, masked=0.2)
    kw = dict(beta=0.25, label_smoothing=0.1, loss_scale=0.5, ref_logp=torch.randn(4, generator=g, device="cuda"))
    d = preference_call(B, x, labels, offsets, **kw)["dlogits"]
    for t, j in [(0, 0), (3, 22), (5, 7), (11, 3), (19, 1)]:
        up, down = x.clone(), x.clone()
        up[t, j] += h
        down[t, j] -= h
        slope = (float(preference_call(B, up, labels, offsets, dlogits=None, **kw)["loss"])
                 - float(preference_call(B, down, labels, offsets, dlogits=None, **kw)["loss"])) / (2 * h)
        assert abs(slope - float(d[t, j])) <= 3e-4, (t, j)


def test_empty_calls(B):
    none = torch.empty(0, device="cuda")
    x, labels = torch.empty((0, 10), device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    B.star_token_logprobs(x, labels, none)
    got = policy_call(B, x, labels, none)
    assert bool((got["sums"] == 0).all())
    got = preference_call(B, x, labels, [0])
    assert bool((got["loss"] == 0).all())
    x, labels = torch.empty((3, 0), device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    got = policy_call(B, x, labels, torch.ones(3, device="cuda"))
    assert bool((got["logp"] == 0).all()) and bool((got["sums"] == 0).all())


def test_other_streams_and_graph_replay(B):
    x, labels, g = make(64, 5000, torch.bfloat16, seed=9)
    A = torch.randn(64, generator=g, device="cuda")
    want = policy_call(B, x, labels, A)
    out = {n: torch.zeros_like(t) for n, t in want.items()}
    ws = torch.empty(B.star_loss_workspace_bytes(64, 4), dtype=torch.uint8, device="cuda")
    offsets = torch.tensor([0, 10, 30, 40, 64], dtype=torch.int32, device="cuda")
    pref = preference_call(B, x, labels, [0, 10, 30, 40, 64])
    pout = {n: torch.zeros_like(t) for n, t in pref.items()}

    def both(stream=None):
        B.star_policy_loss(x, labels, A, out["logp"], out["token_loss"], out["sums"], ws, dlogits=out["dlogits"], stream=stream)
        B.star_preference_loss(x, labels, offsets, pout["seq_logp"], pout["pair_loss"], pout["margin"], pout["loss"], ws,
                               dlogits=pout["dlogits"], stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    both(side)
    side.synchronize()
    for a, b in ((out, want), (pout, pref)):
        for n in b:
            assert torch.equal(a[n], b[n]), n
            a[n].zero_()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        both()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for a, b in ((out, want), (pout, pref)):
        for n in b:
            assert torch.equal(a[n], b[n]), n
