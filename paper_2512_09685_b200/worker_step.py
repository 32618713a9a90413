"""A worker's step in front of the round: from tokens to the gradient buffer that
``star_group_update`` reads.

A small language-model head over frozen token embeddings,

    u = x W1^T,  h = gelu(u),  y = x + h W2^T,  logits = y W3^T,

is trained by the clipped policy loss with a KL term or by the preference loss.
The forward pass keeps the inputs of the three linear layers and of the GELU in
8 bits (``star_checkpoint_pack``; h in the same pass as u's checkpoint); the loss
turns the logits into their gradient in place; the backward pass reads the
checkpoints and writes the three weight gradients straight into the worker's flat
bf16 gradient buffer.  The server's round applies the workers' buffers to the
fp32 master parameters and hands back bf16 snapshots (``star_group_update_ex``),
which are the workers' weights of the next step.

    python -m paper_2512_09685_b200.worker_step [--loss preference] [--rounds N]

plays rounds of four workers on a synthetic task -- after a token t the token
(3 t + 1) mod vocab is rewarded -- and prints the mean reward.  Plain matrix
products are the library's; nothing here computes what the entry points do.
"""
from __future__ import annotations

import argparse
from typing import Dict, List, Optional, Tuple

import torch

from . import binding as B


class HeadWeights:
    """The three weight matrices as views of one flat buffer (any dtype)."""

    def __init__(self, flat: torch.Tensor, d: int, f: int, vocab: int):
        self.flat = flat
        n1, n2 = f * d, d * f
        self.w1 = flat[:n1].view(f, d)
        self.w2 = flat[n1:n1 + n2].view(d, f)
        self.w3 = flat[n1 + n2:].view(vocab, d)

    @staticmethod
    def size(d: int, f: int, vocab: int) -> int:
        return 2 * d * f + vocab * d


class Worker:
    """Buffers of one worker for steps of up to ``rows`` tokens."""

    def __init__(self, rows: int, d: int, f: int, vocab: int, device="cuda"):
        self.rows, self.d, self.f, self.vocab = rows, d, f, vocab
        self.grad = HeadWeights(torch.zeros(HeadWeights.size(d, f, vocab), dtype=torch.bfloat16, device=device), d, f, vocab)
        self.widths = {"x": d, "u": f, "h": f, "y": d}
        self.store = {name: B.star_checkpoint_empty(rows, width, device) for name, width in self.widths.items()}
        self.kept = self.checkpoints(rows)
        self.h = torch.empty((rows, f), dtype=torch.bfloat16, device=device)
        self.logp = torch.empty(rows, device=device)
        self.token_loss = torch.empty(rows, device=device)
        self.sums = torch.empty(4, device=device)
        self.workspace = torch.empty(B.star_loss_workspace_bytes(rows, rows), dtype=torch.uint8, device=device)

    def checkpoints(self, rows: int) -> Dict[str, Tuple[torch.Tensor, torch.Tensor]]:
        """Codes and scales of a step of ``rows`` tokens: the front of the buffers, laid out for that number."""
        kept = {}
        for name, (codes, scales) in self.store.items():
            pitch, code_bytes, scale_bytes = B.star_checkpoint_sizes(rows, self.widths[name])
            kept[name] = (codes.view(-1)[:code_bytes].view(rows, pitch),
                          scales.view(-1)[:scale_bytes].view(scales.shape[0], -1, 4))
        return kept

    def forward(self, x: torch.Tensor, weights: HeadWeights) -> torch.Tensor:
        """Logits of the embeddings x (up to rows x d, bf16); what the backward pass needs is kept in 8 bits."""
        rows = x.shape[0]
        if rows > self.rows:
            raise ValueError("a step of %d tokens, the worker's buffers hold %d" % (rows, self.rows))
        self.kept = self.checkpoints(rows)
        h = self.h[:rows]
        B.star_checkpoint_pack(*self.kept["x"], x)
        u = x @ weights.w1.t()
        B.star_checkpoint_pack(*self.kept["u"], u, act="gelu_tanh", act_out=h)
        B.star_checkpoint_pack(*self.kept["h"], h)
        y = torch.addmm(x, h, weights.w2.t())
        B.star_checkpoint_pack(*self.kept["y"], y)
        return y @ weights.w3.t()

    def backward(self, dlogits: torch.Tensor, weights: HeadWeights) -> None:
        """The weight gradients, into ``self.grad``."""
        B.star_checkpoint_weight_grad(self.grad.w3, dlogits, *self.kept["y"])
        dy = dlogits @ weights.w3
        B.star_checkpoint_weight_grad(self.grad.w2, dy, *self.kept["h"])
        du = dy @ weights.w2
        B.star_checkpoint_act_backward(du, du, *self.kept["u"], "gelu_tanh")
        B.star_checkpoint_weight_grad(self.grad.w1, du, *self.kept["x"])

    def policy_step(self, x: torch.Tensor, labels: torch.Tensor, advantages: torch.Tensor, weights: HeadWeights,
                    old_logp: Optional[torch.Tensor] = None, ref_logp: Optional[torch.Tensor] = None,
                    token_weights: Optional[torch.Tensor] = None, kl_coef: float = 0.0) -> torch.Tensor:
        """One step of the policy loss; returns its four sums."""
        logits = self.forward(x, weights)
        rows = x.shape[0]
        B.star_policy_loss(logits, labels, advantages, self.logp[:rows], self.token_loss[:rows], self.sums, self.workspace,
                           dlogits=logits, weights=token_weights, old_logp=old_logp, ref_logp=ref_logp, kl_coef=kl_coef)
        self.backward(logits, weights)
        return self.sums

    def preference_step(self, x: torch.Tensor, labels: torch.Tensor, seq_offsets: torch.Tensor, weights: HeadWeights,
                        ref_seq_logp: Optional[torch.Tensor] = None, beta: float = 0.1) -> Dict[str, torch.Tensor]:
        """One step of the preference loss, the mean over its pairs; returns its results."""
        pairs = (seq_offsets.numel() - 1) // 2
        out = {"seq_logp": torch.empty(2 * pairs, device=x.device), "pair_loss": torch.empty(pairs, device=x.device),
               "margin": torch.empty(pairs, device=x.device), "loss": torch.empty(1, device=x.device)}
        logits = self.forward(x, weights)
        B.star_preference_loss(logits, labels, seq_offsets, out["seq_logp"], out["pair_loss"], out["margin"], out["loss"],
                               self.workspace, dlogits=logits, ref_logp=ref_seq_logp, beta=beta, loss_scale=1.0 / max(pairs, 1))
        self.backward(logits, weights)
        return out


class Server:
    """fp32 master parameters and momentum, and the bf16 copy that the workers compute with."""

    def __init__(self, d: int, f: int, vocab: int, seed: int = 0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        n = HeadWeights.size(d, f, vocab)
        self.params = torch.randn(n, generator=g, device=device) * 0.05
        self.momentum = torch.zeros(n, device=device)
        self.weights = HeadWeights(self.params.to(torch.bfloat16), d, f, vocab)

    def round(self, workers: List[Worker], group_offsets: List[int], group_members: List[int], lr: float, mu: float = 0.9,
              wd: float = 0.0) -> None:
        """One round over the workers' gradient buffers; the last group's snapshot becomes the workers' weights."""
        groups = len(group_offsets) - 1
        snapshots = [None] * (groups - 1) + [self.weights.flat]
        B.star_group_update_ex(self.params, self.momentum, [w.grad.flat for w in workers], group_offsets, group_members,
                               [lr] * groups, mu, wd, snapshots=snapshots)


def sample(worker: Worker, x: torch.Tensor, weights: HeadWeights, generator) -> Tuple[torch.Tensor, torch.Tensor]:
    """A token per row from the model, and its log-probability."""
    logits = worker.forward(x, weights)
    noise = torch.empty_like(logits, dtype=torch.float32).exponential_(generator=generator).log_()
    labels = (logits.float() - noise).argmax(1)          # the largest of Gumbel-perturbed logits
    logp = torch.empty(x.shape[0], device=x.device)
    B.star_token_logprobs(logits, labels, logp)
    return labels, logp


def play(loss: str = "policy", rounds: int = 40, rows: int = 512, d: int = 64, f: int = 128, vocab: int = 101, n_workers: int = 4,
         lr: Optional[float] = None, seed: int = 0) -> List[float]:
    """Mean reward per round."""
    if lr is None:
        lr = 0.5 if loss == "policy" else 2.0
    g = torch.Generator(device="cuda").manual_seed(seed)
    embeddings = torch.randn((vocab, d), generator=g, device="cuda").to(torch.bfloat16)
    server = Server(d, f, vocab, seed)
    workers = [Worker(rows, d, f, vocab) for _ in range(n_workers)]
    offsets, members = B.star_schedule_static_x(None, n_workers, n_workers)          # all workers' gradients in one update
    ref = HeadWeights(server.weights.flat.clone(), d, f, vocab)
    history = []
    for _ in range(rounds):
        total = 0.0
        for w in workers:
            tokens = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
            wanted = (3 * tokens + 1) % vocab
            x = embeddings[tokens]
            labels, old = sample(w, x, server.weights, g)
            reward = (labels == wanted).float()
            total += float(reward.mean())
            if loss == "policy":
                ref_logp = torch.empty(rows, device="cuda")
                B.star_token_logprobs(w.forward(x, ref), labels, ref_logp)
                # An occasional demonstration keeps a signal while no sample is right.
                shown = torch.rand(rows, generator=g, device="cuda") < 0.25
                labels = torch.where(shown, wanted, labels)
                advantages = torch.where(shown, torch.ones_like(reward), reward - reward.mean())
                w.policy_step(x, labels, advantages, server.weights, None, ref_logp,
                              torch.full((rows,), 1.0 / rows, device="cuda"), kl_coef=1e-3)
            else:
                # Pairs of one-token answers to the same token: the wanted one over the sampled one.
                half = rows // 2
                both = x[:half].repeat_interleave(2, 0).contiguous()
                answers = torch.stack([wanted[:half], labels[:half]], 1).reshape(-1)
                w.preference_step(both, answers, torch.arange(2 * half + 1, dtype=torch.int32, device="cuda"), server.weights,
                                  beta=1.0)
        server.round(workers, offsets, members, lr)
        history.append(total / n_workers)
    B.star_check_waits()
    return history


def main() -> None:
    parser = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    parser.add_argument("--loss", choices=("policy", "preference"), default="policy")
    parser.add_argument("--rounds", type=int, default=40)
    a = parser.parse_args()
    for i, reward in enumerate(play(a.loss, a.rounds)):
        if i % 5 == 0 or i == a.rounds - 1:
            print("round %3d  mean reward %.3f" % (i, reward))


if __name__ == "__main__":
    main()
