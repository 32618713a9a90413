"""A worker's steps of fewer tokens than its buffers hold: the same bits as a
worker made for that number."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 63, 64, 130, 200])
@pytest.mark.parametrize("loss", ["policy", "preference"])
def test_steps_of_any_number_of_tokens(loss, rows):
    from paper_2512_09685_b200 import worker_step as WS
    d, f, vocab, most = 72, 130, 101, 200
    g = torch.Generator(device="cuda").manual_seed(rows)
    server = WS.Server(d, f, vocab, seed=1)
    x = torch.randn((rows, d), generator=g, device="cuda").to(torch.bfloat16)
    labels = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    A = torch.randn(rows, generator=g, device="cuda")
    offsets = torch.tensor([0, rows // 2, rows], dtype=torch.int32, device="cuda")
    results = []
    for size in (most, rows):
        w = WS.Worker(size, d, f, vocab)
        for step in range(2):                              # a longer step's leavings do not matter
            n = size if step == 0 else rows
            if loss == "policy":
                xs, ls, As = [torch.cat([t] * (n // rows + 1))[:n] for t in (x, labels, A)]
                out = w.policy_step(xs, ls, As, server.weights).clone()
            else:
                xs, ls = [torch.cat([t] * (n // rows + 1))[:n] for t in (x, labels)]
                o = offsets if n == rows else torch.tensor([0, n // 3, n], dtype=torch.int32, device="cuda")
                out = torch.cat([v.reshape(-1) for v in w.preference_step(xs, ls, o, server.weights).values()])
        results.append((out, w.grad.flat.clone()))
    assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])
    assert bool(torch.isfinite(results[0][1].float()).all())


def test_more_tokens_than_the_buffers_hold_are_refused():
    from paper_2512_09685_b200 import worker_step as WS
    server = WS.Server(16, 32, 10)
    w = WS.Worker(8, 16, 32, 10)
    with pytest.raises(ValueError):
        w.forward(torch.zeros((9, 16), dtype=torch.bfloat16, device="cuda"), server.weights)


@pytest.mark.parametrize("loss", ["policy", "preference"])
def test_play_with_an_odd_number_of_tokens(loss):
    from paper_2512_09685_b200 import worker_step as WS
    assert len(WS.play(loss, rounds=2, rows=37, d=16, f=24, vocab=11, n_workers=2)) == 2
