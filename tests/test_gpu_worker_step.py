"""A worker's step end to end: gradients through the 8-bit checkpoints against
the same model in binary64, and rounds that learn a task."""
import pytest
import torch

from tests import worker_step_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def WS():
    from paper_2512_09685_b200 import worker_step
    return worker_step


@pytest.mark.parametrize("rows,d,f,vocab", [(200, 64, 128, 101), (97, 40, 72, 1000)])
@pytest.mark.parametrize("loss", ["policy", "preference"])
def test_gradients_against_the_model_in_64_bits(WS, loss, rows, d, f, vocab):
    """Kept values are off by at most 1/254 of their block's largest magnitude
    (0.4 %, about 1 % of a typical value), bf16 intermediates and outputs by 0.4 %
    each: 3 % of the gradient's norm is a generous bound, and a wrong term is far
    beyond it."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    server = WS.Server(d, f, vocab, seed=1)
    w = WS.Worker(rows, d, f, vocab)
    x = torch.randn((rows, d), generator=g, device="cuda").to(torch.bfloat16)
    labels = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    labels[::7] = -100
    flat = server.weights.flat.double().requires_grad_(True)
    m = WS.HeadWeights(flat, d, f, vocab)
    u = x.double() @ m.w1.t()
    logits = (x.double() + R.act(u, "gelu_tanh") @ m.w2.t()) @ m.w3.t()
    lp = torch.where(labels >= 0, torch.log_softmax(logits, 1).gather(1, labels.clamp(min=0)[:, None])[:, 0], torch.zeros((), device="cuda").double())
    if loss == "policy":
        A = torch.randn(rows, generator=g, device="cuda")
        ref = lp.detach().float() + 0.2 * torch.randn(rows, generator=g, device="cuda")
        weights = torch.full((rows,), 1.0 / rows, device="cuda")
        sums = w.policy_step(x, labels, A, server.weights, None, ref, weights, kl_coef=0.1)
        d_ref = ref.double() - lp
        total = (torch.where(labels >= 0, -torch.exp(lp - lp.detach()) * A.double() + 0.1 * (torch.exp(d_ref) - d_ref - 1),
                             torch.zeros_like(lp)) / rows).sum()
        assert abs(float(sums[0]) - float(total.detach())) <= 0.02 * (1 + abs(float(total.detach())))
    else:
        offsets = torch.tensor([0, rows // 5, rows // 2, rows // 2 + 3, rows], dtype=torch.int32, device="cuda")
        out = w.preference_step(x, labels, offsets, server.weights, beta=0.3)
        n = offsets.tolist()
        L = [lp[a:b].sum() for a, b in zip(n, n[1:])]
        total = -(torch.nn.functional.logsigmoid(0.3 * (L[0] - L[1])) + torch.nn.functional.logsigmoid(0.3 * (L[2] - L[3]))) / 2
        # the sums of many log-probabilities: their bf16 logits leave 0.4 % of up to a few hundred
        assert abs(float(out["loss"]) - float(total.detach())) <= 0.05 * (1 + abs(float(total.detach())))
    total.backward()
    want = WS.HeadWeights(flat.grad, d, f, vocab)
    for name in ("w1", "w2", "w3"):
        assert R.rel(getattr(w.grad, name), getattr(want, name)) <= 0.03, name


def test_rounds_learn_the_task(WS):
    from paper_2512_09685_b200 import binding as B
    for loss in ("policy", "preference"):
        before = B.star_launch_count()
        history = WS.play(loss, rounds=40)
        assert history[-1] >= 0.5 and history[0] <= 0.1, (loss, history)
        assert B.star_launch_count() > before + 40 * 4 * 8


def test_check_waits(WS):
    from paper_2512_09685_b200 import binding as B
    B.star_check_waits()
    side = torch.cuda.Stream()
    B.star_check_waits(side)
    with pytest.raises(B.StarError) as e:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            torch.zeros(1, device="cuda")
            B.star_check_waits()
    assert e.value.status == B.STAR_ERR_UNSUPPORTED
