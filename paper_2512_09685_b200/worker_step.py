"""A worker's step in front of the round: from tokens to the gradient buffer that
``star_group_update`` reads.

A small language-model head over frozen token embeddings,

    u = x W1^T,  h = gelu(u),  y = x + h W2^T,  logits = y W3^T,

is trained by the clipped policy loss with a KL term, by the preference loss, or by
distillation from a teacher's recorded top alternatives; then the head reads y
through a root-mean-square norm (``star_rms_norm``).  Its result is kept in 8 bits, for
the head's weight gradient, and y itself in bf16, for the norm's backward pass.
The forward pass keeps the inputs of the three linear layers and of the GELU in
8 bits (``star_checkpoint_pack``; h in the same pass as u's checkpoint); the loss
turns the logits into their gradient in place; the backward pass reads the
checkpoints and writes the three weight gradients straight into the worker's flat
bf16 gradient buffer.  The server's round applies the workers' buffers to the
fp32 master parameters and hands back bf16 snapshots (``star_group_update_ex``),
which are the workers' weights of the next step.

    python -m paper_2512_09685_b200.worker_step [--loss preference|distill] [--rounds N]

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
    """The three weight matrices, and the norm's gain where there is one, as views of one flat buffer (any dtype)."""

    def __init__(self, flat: torch.Tensor, d: int, f: int, vocab: int, norm: bool = False):
        self.flat = flat
        n1, n2, n3 = f * d, d * f, vocab * d
        self.w1 = flat[:n1].view(f, d)
        self.w2 = flat[n1:n1 + n2].view(d, f)
        self.w3 = flat[n1 + n2:n1 + n2 + n3].view(vocab, d)
        self.gain = flat[n1 + n2 + n3:] if norm else None

    @staticmethod
    def size(d: int, f: int, vocab: int, norm: bool = False) -> int:
        return 2 * d * f + vocab * d + (d if norm else 0)


class Worker:
    """Buffers of one worker for steps of up to ``rows`` tokens."""

    def __init__(self, rows: int, d: int, f: int, vocab: int, device="cuda", norm: bool = False):
        self.rows, self.d, self.f, self.vocab = rows, d, f, vocab
        self.grad = HeadWeights(torch.zeros(HeadWeights.size(d, f, vocab, norm), dtype=torch.bfloat16, device=device), d, f, vocab, norm)
        self.widths = {"x": d, "u": f, "h": f, "y": d}
        self.store = {name: B.star_checkpoint_empty(rows, width, device) for name, width in self.widths.items()}
        self.kept = self.checkpoints(rows)
        self.h = torch.empty((rows, f), dtype=torch.bfloat16, device=device)
        self.logp = torch.empty(rows, device=device)
        self.token_loss = torch.empty(rows, device=device)
        self.sums = torch.empty(4, device=device)
        self.workspace = torch.empty(B.star_loss_workspace_bytes(rows, rows), dtype=torch.uint8, device=device)
        self.norm = norm
        if norm:
            # The stream, which the norm's backward pass reads, and its norm, which the head reads in the forward pass.
            self.y, self.normed = (torch.empty((rows, d), dtype=torch.bfloat16, device=device) for _ in range(2))
            self.rstd = torch.empty(rows, device=device)
            self.norm_workspace = torch.empty(B.star_rms_norm_workspace_bytes(rows, d), dtype=torch.uint8, device=device)

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
        if self.norm:
            normed = self.normed[:rows]
            B.star_rms_norm(normed, h @ weights.w2.t(), weights.gain, residual=x, total=self.y[:rows], rstd=self.rstd[:rows],
                            codes=self.kept["y"][0], scales=self.kept["y"][1])
            return normed @ weights.w3.t()
        y = torch.addmm(x, h, weights.w2.t())
        B.star_checkpoint_pack(*self.kept["y"], y)
        return y @ weights.w3.t()

    def backward(self, dlogits: torch.Tensor, weights: HeadWeights) -> None:
        """The weight gradients, into ``self.grad``."""
        B.star_checkpoint_weight_grad(self.grad.w3, dlogits, *self.kept["y"])
        dy = dlogits @ weights.w3
        if self.norm:
            rows = dy.shape[0]
            B.star_rms_norm_backward(dy, self.grad.gain, dy, weights.gain, self.rstd[:rows], self.norm_workspace, total=self.y[:rows])
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

    def distill_step(self, x: torch.Tensor, teacher_ids: torch.Tensor, teacher_logp: torch.Tensor, weights: HeadWeights,
                     labels: Optional[torch.Tensor] = None, token_weights: Optional[torch.Tensor] = None, temperature: float = 1.0,
                     label_coef: float = 0.0) -> torch.Tensor:
        """One step of distillation from a teacher's record (``record``) at the same temperature; returns its four sums."""
        logits = self.forward(x, weights)
        rows = x.shape[0]
        B.star_distillation_loss(logits, teacher_ids, teacher_logp, self.token_loss[:rows], self.sums, self.workspace, dlogits=logits,
                                 labels=labels, weights=token_weights, temperature=temperature, rest=True,
                                 soft_coef=1.0 - label_coef, label_coef=label_coef)
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

    def __init__(self, d: int, f: int, vocab: int, seed: int = 0, device="cuda", norm: bool = False):
        g = torch.Generator(device=device).manual_seed(seed)
        n = HeadWeights.size(d, f, vocab, norm)
        self.params = torch.randn(n, generator=g, device=device) * 0.05
        if norm:
            self.params[-d:] = 1.0
        self.momentum = torch.zeros(n, device=device)
        self.weights = HeadWeights(self.params.to(torch.bfloat16), d, f, vocab, norm)

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


def record(logits: torch.Tensor, k: int, temperature: float = 1.0) -> Tuple[torch.Tensor, torch.Tensor]:
    """What is kept of a teacher's logits: the ids of the k largest of each row and their log-probabilities."""
    ids = torch.empty((logits.shape[0], k), dtype=torch.int32, device=logits.device)
    logp = torch.empty((logits.shape[0], k), device=logits.device)
    B.star_token_alternatives(logits, ids, logp, temperature=temperature)
    return ids, logp


def play(loss: str = "policy", rounds: int = 40, rows: int = 512, d: int = 64, f: int = 128, vocab: int = 101, n_workers: int = 4,
         lr: Optional[float] = None, seed: int = 0) -> List[float]:
    """Mean reward per round."""
    if lr is None:
        lr = {"policy": 0.5, "preference": 2.0, "distill": 0.5}[loss]
    norm = loss == "distill"
    g = torch.Generator(device="cuda").manual_seed(seed)
    embeddings = torch.randn((vocab, d), generator=g, device="cuda").to(torch.bfloat16)
    server = Server(d, f, vocab, seed, norm=norm)
    workers = [Worker(rows, d, f, vocab, norm=norm) for _ in range(n_workers)]
    offsets, members = B.star_schedule_static_x(None, n_workers, n_workers)          # all workers' gradients in one update
    ref = HeadWeights(server.weights.flat.clone(), d, f, vocab, norm)
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
            elif loss == "distill":
                # A teacher that is fairly sure of the wanted token, and of the rest as it comes.
                teacher = torch.randn((rows, vocab), generator=g, device="cuda")
                teacher.scatter_(1, wanted[:, None], 8.0)
                w.distill_step(x, *record(teacher.to(torch.bfloat16), 8), server.weights, wanted,
                               torch.full((rows,), 1.0 / rows, device="cuda"), label_coef=0.25)
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
    parser.add_argument("--loss", choices=("policy", "preference", "distill"), default="policy")
    parser.add_argument("--rounds", type=int, default=40)
    a = parser.parse_args()
    for i, reward in enumerate(play(a.loss, a.rounds)):
        if i % 5 == 0 or i == a.rounds - 1:
            print("round %3d  mean reward %.3f" % (i, reward))


if __name__ == "__main__":
    main()
