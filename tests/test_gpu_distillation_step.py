"""A teacher's record, a worker's distillation step through the norm, and the round
behind it, run together; the same in captured graphs, on other streams, and twice at
once."""
import math

import pytest
import torch

from . import distillation_reference as R

pytestmark = pytest.mark.gpu
ROWS, D, F, V, K = 96, 64, 128, 501, 9


def gpu(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def setup(rows=ROWS, seed=0):
    from paper_2512_09685_b200 import worker_step as W
    server, worker = W.Server(D, F, V, seed, norm=True), W.Worker(ROWS, D, F, V, norm=True)
    g = gpu(seed + 1)
    server.weights.gain.copy_((1 + 0.1 * torch.randn(D, generator=g, device="cuda")).to(torch.bfloat16))
    x = torch.randn((rows, D), generator=g, device="cuda").to(torch.bfloat16)
    teacher = (3 * torch.randn((rows, V), generator=g, device="cuda")).to(torch.bfloat16)
    labels = torch.randint(0, V, (rows,), generator=g, device="cuda")
    labels[::5] = -100
    weights = torch.rand(rows, generator=g, device="cuda") / rows
    return W, server, worker, x, teacher, labels, weights


def restored(kept, rows, cols):
    from paper_2512_09685_b200 import binding as B
    out = torch.empty((rows, cols), device="cuda")
    B.star_checkpoint_unpack(out, *kept)
    return out.double()


def relative(got, want):
    return float((got.double() - want).norm() / want.norm())


def test_each_stage_of_a_step_against_its_formula():
    W, server, worker, x, teacher, labels, weights = setup()
    ids, logp = W.record(teacher, K)
    want = R.alternatives(teacher, K)
    assert torch.equal(ids.long(), want["ids"])
    sums = worker.distill_step(x, ids, logp, server.weights, labels, weights, label_coef=0.25)
    weight, grad = server.weights, worker.grad
    # The forward pass: what the worker kept of it, each from what it kept of the stage in front.
    y, rstd = worker.y, worker.rstd
    normed, r = R.norm(y, weight.gain, 1e-6)
    assert relative(worker.normed, normed) <= R.half_step(torch.bfloat16) and relative(rstd, r) <= R.norm_bound(D)
    codes = restored(worker.kept["y"], ROWS, D)
    assert float((codes - worker.normed.double()).abs().max()) <= float(worker.normed.abs().max()) / 127
    logits = (worker.normed @ weight.w3.t())
    loss = R.distillation(logits, ids, logp, labels, weights, rest=True, soft=0.75, hard=0.25)
    assert bool(((worker.token_loss.double() - loss["token_loss"]).abs() <= loss["token_bound"]).all())
    assert bool(((sums.double() - loss["sums"]).abs() <= loss["sums_bound"]).all())
    # The backward pass, from the gradient of the logits rounded to bf16 as the step rounds it.
    half = R.half_step(torch.bfloat16)
    dlogits = loss["dlogits"]
    assert relative(grad.w3, dlogits.t() @ codes) <= 4 * half
    dnormed = (dlogits.to(torch.bfloat16) @ weight.w3).to(torch.bfloat16)
    dy, dgain, _, _ = R.norm_backward(dnormed, y, rstd, weight.gain)
    assert relative(grad.gain, dgain) <= 4 * half
    assert relative(grad.w2, dy.t() @ restored(worker.kept["h"], ROWS, F)) <= 4 * half


def test_the_gradients_are_those_of_the_loss():
    """The whole step against automatic differentiation of its formulas; 8-bit and bf16 steps between them leave a few per cent."""
    W, server, worker, x, teacher, labels, weights = setup(seed=3)
    ids, logp = W.record(teacher, K)
    worker.distill_step(x, ids, logp, server.weights, labels, weights, label_coef=0.25)
    leaf = server.weights.flat.double().requires_grad_(True)
    w = W.HeadWeights(leaf, D, F, V, True)
    u = x.double() @ w.w1.t()
    h = torch.nn.functional.gelu(u, approximate="tanh")
    y = x.double() + h @ w.w2.t()
    normed = y / torch.sqrt(y.square().mean(1, keepdim=True) + 1e-6) * w.gain
    every = torch.log_softmax(normed @ w.w3.t(), 1)
    q = logp.double().exp()
    q0 = 1 - q.sum(1)
    listed = torch.zeros_like(every, dtype=torch.bool).scatter_(1, ids.long(), True)
    apart = torch.logsumexp(every.masked_fill(listed, -math.inf), 1)
    kl = (q * (logp.double() - every.gather(1, ids.long()))).sum(1) + q0 * (q0.log() - apart)
    ce = -every.gather(1, labels.clamp(min=0)[:, None])[:, 0]
    (torch.where(labels >= 0, weights.double(), torch.zeros_like(kl)) * (0.75 * kl + 0.25 * ce)).sum().backward()
    want = W.HeadWeights(leaf.grad, D, F, V, True)
    for name in ("w1", "w2", "w3", "gain"):
        assert relative(getattr(worker.grad, name), getattr(want, name)) <= 0.05, name


def test_shorter_steps_and_rounds():
    W, server, worker, x, teacher, labels, weights = setup(rows=37, seed=5)
    ids, logp = W.record(teacher, K)
    sums = worker.distill_step(x, ids, logp, server.weights, labels, weights)
    again = W.Worker(37, D, F, V, norm=True)
    sums2 = again.distill_step(x, ids, logp, server.weights, labels, weights)
    assert torch.equal(sums, sums2) and torch.equal(worker.grad.flat, again.grad.flat)
    before = server.params.clone()
    server.round([worker, again], [0, 2], [0, 1], 0.1)
    assert torch.equal(server.weights.flat, server.params.to(torch.bfloat16)) and not torch.equal(before, server.params)


def test_it_runs():
    from paper_2512_09685_b200 import worker_step as W
    history = W.play("distill", rounds=3, rows=64)
    assert len(history) == 3 and all(0.0 <= r <= 1.0 for r in history)


def test_a_captured_step_replays_with_new_inputs():
    """Two graphs and eager steps take turns; each result is that of an eager step on the same inputs."""
    W, server, worker, x, teacher, labels, weights = setup(seed=7)
    ids, logp = torch.empty((ROWS, K), dtype=torch.int32, device="cuda"), torch.empty((ROWS, K), device="cuda")
    from paper_2512_09685_b200 import binding as B

    def step(w):
        B.star_token_alternatives(teacher, ids, logp)
        return w.distill_step(x, ids, logp, server.weights, labels, weights, label_coef=0.5)

    stream = torch.cuda.Stream()
    others = [W.Worker(ROWS, D, F, V, norm=True) for _ in range(2)]
    graphs = []
    with torch.cuda.stream(stream):
        for w in others:
            step(w)                                            # the libraries' own start
        stream.synchronize()
        for w in others:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                step(w)
            graphs.append(graph)
        for seed in range(3):
            teacher.copy_((3 * torch.randn((ROWS, V), generator=gpu(seed), device="cuda")).to(torch.bfloat16))
            weights.copy_(torch.rand(ROWS, generator=gpu(seed + 9), device="cuda"))
            for graph in graphs:
                graph.replay()
            step(worker)
            stream.synchronize()
            for w in others:
                assert torch.equal(w.grad.flat, worker.grad.flat) and torch.equal(w.sums, worker.sums)
    B.star_check_waits()


def test_two_steps_at_once():
    """Workers with buffers of their own on two streams, many times over."""
    W, server, worker, x, teacher, labels, weights = setup(seed=9)
    ids, logp = W.record(teacher, K)
    worker.distill_step(x, ids, logp, server.weights, labels, weights, label_coef=0.5)
    torch.cuda.synchronize()
    workers = [W.Worker(ROWS, D, F, V, norm=True) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in workers]
    for _ in range(20):
        for w, s in zip(workers, streams):
            with torch.cuda.stream(s):
                w.distill_step(x, ids, logp, server.weights, labels, weights, label_coef=0.5)
    torch.cuda.synchronize()
    for w in workers:
        assert torch.equal(w.grad.flat, worker.grad.flat) and torch.equal(w.sums, worker.sums)


@pytest.mark.parametrize("rows,vocab", [(3, 70001), (400, 3001), (5, 900)])
def test_operators_follow_one_another_without_a_wait_between(rows, vocab):
    """Each reads what the kernel in front has just written, on one stream; the same call by call with waits."""
    from paper_2512_09685_b200 import binding as B
    g = gpu(rows)
    k = 20
    x = (2 * torch.randn((rows, vocab), generator=g, device="cuda")).to(torch.bfloat16)
    labels = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    ones = torch.ones(rows, device="cuda")

    def chain(wait):
        sync = torch.cuda.synchronize if wait else lambda: None
        ids, top = torch.empty((rows, k), dtype=torch.int32, device="cuda"), torch.empty((rows, k), device="cuda")
        lse, entropy = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        d, loss, sums = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(4, device="cuda")
        ws = torch.empty(B.star_loss_workspace_bytes(rows), dtype=torch.uint8, device="cuda")
        ws2 = torch.empty(B.star_rms_norm_workspace_bytes(rows, vocab), dtype=torch.uint8, device="cuda")
        y, rstd, dgain = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(vocab, device="cuda")
        out = []
        for _ in range(3):
            B.star_token_alternatives(x, ids, top, labels=labels, lse=lse, entropy=entropy)
            sync()
            B.star_token_alternatives_backward(d, x, lse, labels=labels, d_logp=ones, entropy=entropy, d_entropy=ones, top_ids=ids, d_top_logp=top)
            sync()
            B.star_distillation_loss(d, ids, top, loss, sums, ws, dlogits=d, rest=True)
            sync()
            B.star_rms_norm(y, d, None, rstd=rstd)
            sync()
            B.star_rms_norm_backward(d, dgain, d, None, rstd, ws2, total=y)
            sync()
            out += [t.clone() for t in (ids, top, lse, loss, sums, d, dgain, rstd)]
        torch.cuda.synchronize()
        return out

    assert all(torch.equal(p, q) for p, q in zip(chain(False), chain(True)))
