"""Order in a stream.  The operators' blocks may be set up while the kernel in
front is still running; what they read and write must be as if they were not.
Everything is compared for equality with the same calls one by one, each waited
for."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2512_09685_b200 import binding
    return binding


class Step:
    """A chain in which every call reads what the one in front of it wrote, or overwrites what that one reads."""

    def __init__(self, B, T, C, V, dtype):
        self.B, self.T, self.C, self.V = B, T, C, V
        new = lambda *s, dt=torch.float32: torch.zeros(s, device="cuda", dtype=dt)  # noqa: E731
        self.source = torch.randn((4, T, max(C, V)), device="cuda").to(dtype)
        self.x, self.h, self.logits, self.dlogits = new(T, C, dt=dtype), new(T, C, dt=dtype), new(T, V, dt=dtype), new(T, V, dt=dtype)
        self.codes, self.scales = B.star_checkpoint_empty(T, C)
        self.labels = torch.randint(0, V, (T,), device="cuda")
        self.A, self.old, self.lp, self.tl, self.sums = torch.randn(T, device="cuda"), new(T), new(T), new(T), new(4)
        self.ws = torch.empty(B.star_loss_workspace_bytes(T, 2), dtype=torch.uint8, device="cuda")
        self.dw, self.total = new(V, C), new(V, C)

    def run(self, i, wait=lambda: None):
        B = self.B
        steps = [
            lambda: self.x.copy_(self.source[i, :, :self.C]),
            lambda: B.star_checkpoint_pack(self.codes, self.scales, self.x, act="gelu_tanh", act_out=self.h),
            lambda: B.star_checkpoint_unpack(self.x, self.codes, self.scales),                    # overwrites what the pack reads
            lambda: self.logits.copy_(self.source[(i + 1) % 4, :, :self.V]),
            lambda: B.star_token_logprobs(self.logits, self.labels, self.old),
            lambda: self.logits.mul_(1.25),                                                       # overwrites what the logprobs read
            lambda: B.star_policy_loss(self.logits, self.labels, self.A, self.lp, self.tl, self.sums, self.ws,
                                       dlogits=self.dlogits, old_logp=self.old, kl_coef=0.1),
            lambda: B.star_checkpoint_weight_grad(self.dw, self.dlogits, self.codes, self.scales),
            lambda: self.total.add_(self.dw),
            lambda: B.star_checkpoint_weight_grad(self.dw, self.logits, self.codes, self.scales, accumulate=True),
            lambda: B.star_checkpoint_act_backward(self.h, self.x, self.codes, self.scales, "silu"),
            lambda: B.star_checkpoint_pack(self.codes, self.scales, self.h),                      # overwrites what that reads
            lambda: B.star_policy_loss(self.logits, self.labels, self.A, self.lp, self.tl, self.sums, self.ws, dlogits=self.logits),
            lambda: self.total.add_(self.dw),
        ]
        for step in steps:
            step()
            wait()

    def results(self):
        return [t.clone() for t in (self.codes, self.scales, self.x, self.h, self.logits, self.dlogits, self.old, self.lp,
                                    self.tl, self.sums, self.dw, self.total)]


SIZES = [(16, 64, 100), (130, 256, 1000), (600, 512, 2050), (2048, 1024, 4096)]


def one_by_one(step, n):
    step.total.zero_()
    for i in range(n):
        step.run(i % 4, torch.cuda.synchronize)
    return step.results()


def same(got, want):
    return all(torch.equal(g, w) or torch.equal(torch.isnan(g.float()), torch.isnan(w.float())) and
               torch.equal(torch.nan_to_num(g.float()), torch.nan_to_num(w.float())) for g, w in zip(got, want))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,C,V", SIZES)
def test_calls_in_a_row(B, T, C, V, dtype):
    torch.manual_seed(T)
    step = Step(B, T, C, V, dtype)
    want = one_by_one(step, 3)
    for _ in range(4):
        step.total.zero_()
        for i in range(3):
            step.run(i)
        torch.cuda.synchronize()
        assert same(step.results(), want)


@pytest.mark.parametrize("T,C,V", SIZES[1:3])
def test_streams_that_take_turns(B, T, C, V):
    torch.manual_seed(T)
    step = Step(B, T, C, V, torch.bfloat16)
    want = one_by_one(step, 6)
    step.total.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for i in range(6):
        here, other = streams[i % 2], streams[1 - i % 2]
        here.wait_stream(other)
        with torch.cuda.stream(here):
            step.run(i % 4)
    torch.cuda.synchronize()
    assert same(step.results(), want)


@pytest.mark.parametrize("T,C,V", SIZES[1:3])
def test_in_a_graph(B, T, C, V):
    """Behind copies, behind a fill, behind a join of two branches, and first in a graph."""
    torch.manual_seed(T)
    step = Step(B, T, C, V, torch.bfloat16)
    want = one_by_one(step, 2)
    first = torch.zeros(T, device="cuda")
    B.star_token_logprobs(step.logits, step.labels, first)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    at_start, behind_fill, behind_join = torch.zeros(T, device="cuda"), torch.ones(T, device="cuda"), torch.ones(T, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.star_token_logprobs(step.logits, step.labels, at_start)
        step.total.zero_()
        step.run(0)
        step.run(1)
        behind_fill.zero_()
        B.star_token_logprobs(step.logits, step.labels, behind_fill)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other = step.logits.clone()
        behind_join.zero_()
        torch.cuda.current_stream().wait_stream(side)
        B.star_token_logprobs(other, step.labels, behind_join)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert same(step.results(), want)
        assert torch.equal(at_start, first) and torch.equal(behind_fill, first) and torch.equal(behind_join, first)
