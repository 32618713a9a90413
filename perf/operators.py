"""What is measured of the operators of a worker's step: the losses over the
vocabulary with their gradients, and activations kept in 8 bits with their use
in the backward pass.

``run`` is a user's pass through an operator (``own``) or the same result from
elementary torch operations in 32 bits; ``exact`` is the definition in 64 bits.
"""
import math

import torch

own = False

GPT2_VOCAB = 50257
BF16, F32 = "bf16", "f32"
TORCH_TYPE = {BF16: torch.bfloat16, F32: torch.float32}
SIZE = {BF16: 2, F32: 4}

CLIP_LOW, CLIP_HIGH, KL = 0.2, 0.25, 0.05
BETA, SMOOTHING = 0.1, 0.05


def listed():
    return [
        # One micro-batch of a policy update: 8 sequences of 1024 tokens, a third of them prompt.
        dict(name="policy 8x1024 tokens", op="policy", rows=8192, vocab=GPT2_VOCAB, dtype=BF16, masked=0.35, ref=True, grad=True),
        # The last, short completion of an epoch, logits kept in fp32.
        dict(name="policy 37 tokens fp32", op="policy", rows=37, vocab=32001, dtype=F32, masked=0.2, ref=True, grad=True),
        # A micro-batch of eight answer pairs of up to 512 tokens each.
        dict(name="preference 8 pairs", op="preference", pairs=8, longest=512, vocab=GPT2_VOCAB, dtype=BF16, ref=True, average=False),
        # A single pair of one-line answers.
        dict(name="preference 1 short pair", op="preference", pairs=1, longest=24, vocab=GPT2_VOCAB, dtype=BF16, ref=True, average=True),
        # Old and reference log-probabilities of a rollout.
        dict(name="logprobs 4096 tokens", op="logprobs", rows=4096, vocab=GPT2_VOCAB, dtype=BF16, masked=0.3),
        # The log-probability of one sampled token.
        dict(name="logprobs 1 token", op="logprobs", rows=1, vocab=GPT2_VOCAB, dtype=BF16, masked=0.0),
        # A GPT-2-medium MLP of 16 sequences: GELU forward, its input kept in 8 bits; and the restored input.
        dict(name="keep 16384x4096", op="keep", rows=16384, cols=4096, dtype=BF16, act="gelu_tanh"),
        # An odd width in fp32.
        dict(name="keep 300x1001 fp32", op="keep", rows=300, cols=1001, dtype=F32, act="silu"),
        # The backward pass of the same GELU.
        dict(name="act backward 16384x4096", op="act_backward", rows=16384, cols=4096, dtype=BF16, act="gelu_tanh"),
        # A short sequence through BERT's GELU in fp32.
        dict(name="act backward 129x4096 fp32", op="act_backward", rows=129, cols=4096, dtype=F32, act="gelu_erf"),
        # Weight gradient of the GPT-2-medium MLP's first linear layer over 16 sequences.
        dict(name="weight grad 16384 tokens", op="weight_grad", rows=16384, cols=1024, outs=4096, dtype=BF16, out_dtype=BF16),
        # Weight gradient of a projection over one short sequence.
        dict(name="weight grad 515 tokens", op="weight_grad", rows=515, cols=1024, outs=1024, dtype=BF16, out_dtype=BF16),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _width(rng, low, high):
    """A layer's width: mostly a multiple of 8, sometimes any number."""
    w = _spread(rng, low, high)
    return w if rng.random() < 0.3 else max(8, w // 8 * 8)


def draw(rng):
    op = rng.choice(["policy", "preference", "logprobs", "keep", "act_backward", "weight_grad"])
    dtype = rng.choice([BF16, BF16, BF16, F32])
    if op in ("policy", "logprobs", "preference"):
        vocab = _spread(rng, 2000, 131072)
        if rng.random() < 0.5:
            vocab = vocab // 64 * 64
        most = 8192 * GPT2_VOCAB * 2 // (vocab * SIZE[dtype])
        if op == "preference":
            pairs = _spread(rng, 1, 16)
            longest = min(_spread(rng, 8, 1024), max(8, most // 4 // pairs))
            return dict(op=op, pairs=pairs, longest=longest, vocab=vocab, dtype=dtype, ref=rng.random() < 0.8, average=rng.random() < 0.3)
        rows = min(_spread(rng, 1, 16384), most)
        masked = round(rng.uniform(0.0, 0.6), 2)
        if op == "logprobs":
            return dict(op=op, rows=rows, vocab=vocab, dtype=dtype, masked=masked)
        return dict(op=op, rows=rows, vocab=vocab, dtype=dtype, masked=masked, ref=rng.random() < 0.7, grad=rng.random() < 0.9)
    act = rng.choice(["gelu_tanh", "gelu_erf", "silu"])
    if op == "weight_grad":
        rows, cols, outs = _spread(rng, 1, 16384), _width(rng, 64, 8192), _width(rng, 64, 8192)
        while 2 * rows * cols * outs > 2 * 16384 * 1024 * 4096:
            rows = rows // 2 + 1
        cols, outs = cols + (cols == 3072), outs + (outs == 3072)
        return dict(op=op, rows=rows, cols=cols, outs=outs, dtype=dtype, out_dtype=F32 if dtype == F32 else rng.choice([BF16, BF16, F32]))
    rows, cols = _spread(rng, 1, 16384), _width(rng, 64, 8192)
    cols = cols + (cols == 3072)
    rows = min(rows, 16384 * 4096 * 2 // (cols * SIZE[dtype]))
    return dict(op=op, rows=rows, cols=cols, dtype=dtype, act=act if op == "act_backward" or rng.random() < 0.6 else "none")


def work(case):
    s = SIZE[case["dtype"]]
    op = case["op"]
    if op in ("policy", "logprobs", "preference"):
        rows = sum(_lengths(case)) if op == "preference" else case["rows"]
        read = rows - _masked_rows(case, rows)      # masked rows' logits are not needed
        write = rows if op == "preference" or case.get("grad") else 0
        passes = 4 if write else 2                  # exp and sum, then exp and product
        return {"bytes": (read + write) * case["vocab"] * s + 32 * rows, "flops": passes * read * case["vocab"]}
    n = case["rows"] * case["cols"]
    kept = n + n / 32
    if op == "keep":
        return {"bytes": n * s + 2 * kept + n * s * (1 if case["act"] == "none" else 2), "flops": 12 * n}
    if op == "act_backward":
        return {"bytes": 2 * n * s + kept, "flops": 16 * n}
    return {"bytes": kept + case["rows"] * case["outs"] * s + case["cols"] * case["outs"] * SIZE[case["out_dtype"]],
            "flops": 2 * n * case["outs"]}


# --------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------
def _lengths(case):
    """Tokens of each sequence (chosen, rejected, chosen, ...): between a fifth of the longest and the longest."""
    longest, out = case["longest"], []
    for s in range(2 * case["pairs"]):
        out.append(max(1, longest - (s * 7919 + 13 * longest) % (longest * 4 // 5 + 1)))
    return out


def _masked_rows(case, rows):
    if case["op"] == "preference":
        return sum(n // 4 for n in _lengths(case))  # the prompt's tokens, at the front of each sequence
    return int(rows * case["masked"])


def _logits(gen, rows, vocab, dtype):
    """Logits of a language model and labels: the label's log-probability is about -exponential(1.3)."""
    x = torch.empty((rows, vocab), dtype=TORCH_TYPE[dtype], device="cuda")
    labels = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    logp = torch.empty(rows, device="cuda")
    step = max(1, (1 << 26) // vocab)
    for a in range(0, rows, step):
        b = min(rows, a + step)
        z = torch.empty((b - a, vocab), device="cuda").normal_(0.0, 2.0, generator=gen)
        want = torch.empty(b - a, device="cuda").exponential_(1 / 1.3, generator=gen).clamp_(0.02, 12.0)
        rest = torch.logsumexp(z, 1)
        z.scatter_(1, labels[a:b, None], (rest - torch.log(torch.expm1(want)))[:, None])
        x[a:b] = z
        z = x[a:b].float()
        logp[a:b] = z.gather(1, labels[a:b, None])[:, 0] - torch.logsumexp(z, 1)
    return x, labels, logp


def _kept(x):
    """Codes and scales of x as the framework lays them out: int8 [rows, cols rounded up to 16], and a byte e + 127 for every 32
    columns of a row, four of them (128 columns) side by side: [ceil(cols / 128), rows rounded up to 64, 4]."""
    rows, cols = x.shape
    tiles = (cols + 127) // 128
    wide = torch.zeros((rows, tiles * 128), device=x.device)
    wide[:, :cols] = x.float()
    blocks = wide.view(rows, tiles * 4, 32)
    e = _exponent(blocks.abs().amax(2))
    codes = torch.round(blocks * torch.exp2(-e)[:, :, None]).to(torch.int8).view(rows, tiles * 128)
    scales = torch.ones((tiles, (rows + 63) // 64 * 64, 4), dtype=torch.uint8, device=x.device)
    scales[:, :rows] = (e + 127).to(torch.uint8).view(rows, tiles, 4).transpose(0, 1)
    return codes[:, :(cols + 15) // 16 * 16].contiguous(), scales


def _exponent(largest):
    """The smallest e (at least -126) for which the largest magnitude of a block rounds to at most 127 at 2^e."""
    bits = largest.contiguous().view(torch.int32)
    return (((bits + 0x10000) >> 23) - 6).clamp(min=1).float() - 127


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    s = {"case": case}
    if op in ("policy", "logprobs", "preference"):
        lengths = _lengths(case) if op == "preference" else None
        rows = sum(lengths) if lengths else case["rows"]
        x, labels, logp = _logits(gen, rows, case["vocab"], case["dtype"])
        s.update(logits=x, labels=labels, logp=torch.empty(rows, device="cuda"))
        if op == "preference":
            prompt, start = [], 0
            for n in lengths:
                prompt += range(start, start + n // 4)
                start += n
            if prompt:
                labels[torch.tensor(prompt, device="cuda")] = -100
            offsets = [0]
            for n in lengths:
                offsets.append(offsets[-1] + n)
            s["offsets"] = torch.tensor(offsets, dtype=torch.int32, device="cuda")
            # What a training loop keeps of the batch's layout beside the offsets.
            s["sequence"] = torch.repeat_interleave(torch.arange(len(lengths), device="cuda"), torch.tensor(lengths, device="cuda"))
            member = (torch.arange(len(lengths), device="cuda")[:, None] == s["sequence"]) & (labels >= 0)
            total = torch.where(member, logp, torch.zeros_like(logp)).sum(1)
            if case["average"]:
                total = total / member.sum(1).clamp(min=1)
            apart = (0.5 if case["average"] else 8.0) * torch.randn(len(lengths), generator=gen, device="cuda")
            s["ref"] = total + apart if case["ref"] else None
            P = case["pairs"]
            s.update(seq_logp=torch.empty(2 * P, device="cuda"), pair_loss=torch.empty(P, device="cuda"),
                     margin=torch.empty(P, device="cuda"), loss=torch.empty(1, device="cuda"), dlogits=torch.empty_like(x))
        else:
            k = _masked_rows(case, rows)
            drop = torch.randperm(rows, generator=gen, device="cuda")[:k]
            labels[drop] = -100
            s["lse"] = torch.empty(rows, device="cuda")
        if op == "policy":
            shift = 0.15 * torch.randn(rows, generator=gen, device="cuda")
            # No ratio within rounding of the clip's edges: which side such a token falls on is no property of an implementation.
            for edge in (math.log(1 - CLIP_LOW), math.log(1 + CLIP_HIGH)):
                shift = torch.where((shift - edge).abs() < 1e-3, shift + 4e-3, shift)
            s.update(old=logp - shift, ref=logp + 0.3 * torch.randn(rows, generator=gen, device="cuda") if case["ref"] else None,
                     advantages=torch.randn(rows, generator=gen, device="cuda"),
                     weights=(labels >= 0).float() / max(1, rows - k),
                     token_loss=torch.empty(rows, device="cuda"), sums=torch.empty(4, device="cuda"),
                     dlogits=torch.empty_like(x) if case["grad"] else None)
        s["workspace"] = torch.empty((1 << 20) + 32 * rows, dtype=torch.uint8, device="cuda")
        return s
    rows, cols, t = case["rows"], case["cols"], TORCH_TYPE[case["dtype"]]
    # Activations: Gaussian, with a few columns that are ten times as large.
    x = torch.randn((rows, cols), generator=gen, device="cuda")
    x *= 1 + 9 * (torch.rand(cols, generator=gen, device="cuda") < 0.01).float()
    if op == "keep":
        x = x.to(t)
        pitch, tiles, tall = (cols + 15) // 16 * 16, (cols + 127) // 128, (rows + 63) // 64 * 64
        s.update(x=x, codes=torch.empty((rows, pitch), dtype=torch.int8, device="cuda"),
                 scales=torch.empty((tiles, tall, 4), dtype=torch.uint8, device="cuda"),
                 value=torch.empty_like(x) if case["act"] != "none" else None, restored=torch.empty_like(x))
        return s
    s["codes"], s["scales"] = _kept(x.to(t))
    del x
    wide = case["outs"] if op == "weight_grad" else cols
    dy = torch.randn((rows, wide), generator=gen, device="cuda")
    s["dy"] = (dy * 1e-3).to(t)
    if op == "act_backward":
        s["dx"] = torch.empty_like(s["dy"])
    else:
        s["dw"] = torch.empty((case["outs"], cols), dtype=TORCH_TYPE[case["out_dtype"]], device="cuda")
    return s


# --------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------
def run(s):
    return (_own if own else _plain)(s["case"], s)


def _own(case, s):
    from paper_2512_09685_b200 import binding as star
    op = case["op"]
    if op == "logprobs":
        star.star_token_logprobs(s["logits"], s["labels"], s["logp"], s["lse"])
        return s["logp"], s["lse"]
    if op == "policy":
        star.star_policy_loss(s["logits"], s["labels"], s["advantages"], s["logp"], s["token_loss"], s["sums"], s["workspace"],
                              dlogits=s["dlogits"], weights=s["weights"], old_logp=s["old"], ref_logp=s["ref"],
                              clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coef=KL if case["ref"] else 0.0)
        return {"logp": s["logp"], "token_loss": s["token_loss"], "sums": s["sums"], "dlogits": s["dlogits"]}
    if op == "preference":
        star.star_preference_loss(s["logits"], s["labels"], s["offsets"], s["seq_logp"], s["pair_loss"], s["margin"], s["loss"],
                                  s["workspace"], dlogits=s["dlogits"], ref_logp=s["ref"], beta=BETA, label_smoothing=SMOOTHING,
                                  average=case["average"], loss_scale=1.0 / case["pairs"])
        return {"seq_logp": s["seq_logp"], "pair_loss": s["pair_loss"], "margin": s["margin"], "loss": s["loss"], "dlogits": s["dlogits"]}
    if op == "keep":
        star.star_checkpoint_pack(s["codes"], s["scales"], s["x"], act=case["act"], act_out=s["value"])
        star.star_checkpoint_unpack(s["restored"], s["codes"], s["scales"])
        return {"restored": s["restored"], "value": s["value"]}
    if op == "act_backward":
        star.star_checkpoint_act_backward(s["dx"], s["dy"], s["codes"], s["scales"], act=case["act"])
        return s["dx"]
    star.star_checkpoint_weight_grad(s["dw"], s["dy"], s["codes"], s["scales"])
    return s["dw"]


def _row_logp(x, labels):
    z = x.float()
    active = (labels >= 0) & (labels < x.shape[1])
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    at = torch.where(active, labels, torch.zeros_like(labels))
    logp = torch.where(active, z.gather(1, at[:, None])[:, 0] - lse, torch.zeros_like(lse))
    return e, total, active, at, logp, torch.where(active, lse, torch.zeros_like(lse))


def _row_grad(e, total, at, coef, dtype):
    """coef * (onehot - softmax), rounded once."""
    g = e.mul_(-coef[:, None] / total)
    g.scatter_add_(1, at[:, None], coef[:, None])
    return g.to(dtype)


def _slope(x, act):
    if act == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * (x + 0.044715 * x * x * x))
        return 0.5 * (1 + t) + 0.5 * x * (1 - t * t) * k * (1 + 3 * 0.044715 * x * x)
    if act == "gelu_erf":
        return 0.5 * (1 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)
    if act == "silu":
        q = 1 / (1 + torch.exp(-x))
        return q * (1 + x * (1 - q))
    return torch.ones_like(x)


def _act(x, act):
    if act == "gelu_tanh":
        return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x)))
    if act == "gelu_erf":
        return 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))
    if act == "silu":
        return x / (1 + torch.exp(-x))
    return x


def _restore(codes, scales, cols):
    rows = codes.shape[0]
    e = scales[:, :rows].transpose(0, 1).reshape(rows, -1).float() - 127
    step = torch.exp2(e).repeat_interleave(32, 1)[:, :cols]
    return codes[:, :cols].float() * step


def _plain(case, s):
    op = case["op"]
    if op == "logprobs":
        _, _, _, _, logp, lse = _row_logp(s["logits"], s["labels"])
        return logp, lse
    if op == "policy":
        e, total, active, at, logp, _ = _row_logp(s["logits"], s["labels"])
        w = torch.where(active, s["weights"], torch.zeros_like(logp))
        a = s["advantages"]
        r = torch.exp(logp - s["old"])
        u, c = r * a, torch.clamp(r, 1 - CLIP_LOW, 1 + CLIP_HIGH) * a
        gain = torch.minimum(u, c)
        slope = torch.where(u <= c, -u, torch.zeros_like(u))
        kl = torch.zeros_like(u)
        if case["ref"]:
            d = s["ref"] - logp
            kl = torch.exp(d) - d - 1
            slope = slope + KL * (1 - torch.exp(d))
        on = w != 0
        zero = torch.zeros_like(u)
        loss = torch.where(on, -gain + (KL if case["ref"] else 0.0) * kl, zero)
        sums = torch.stack([(w * loss).sum(), (w * torch.where(on, -gain, zero)).sum(), (w * torch.where(on, kl, zero)).sum(),
                            (w * (u > c).float()).sum()])
        grad = _row_grad(e, total, at, w * torch.where(on, slope, zero), s["logits"].dtype) if case["grad"] else None
        return {"logp": logp, "token_loss": loss, "sums": sums, "dlogits": grad}
    if op == "preference":
        e, total, active, at, logp, _ = _row_logp(s["logits"], s["labels"])
        P = case["pairs"]
        member = torch.arange(2 * P, device=logp.device)[:, None] == s["sequence"]
        seq = torch.where(member, logp, torch.zeros_like(logp)).sum(1)
        count = torch.ones_like(seq)
        if case["average"]:
            count = (member & active).float().sum(1).clamp(min=1)
            seq = seq / count
        h = seq[0::2] - seq[1::2]
        if case["ref"]:
            h = h - (s["ref"][0::2] - s["ref"][1::2])
        bh = BETA * h
        softplus = torch.log1p(torch.exp(-bh.abs()))
        pair = (1 - SMOOTHING) * (softplus + (-bh).clamp(min=0)) + SMOOTHING * (softplus + bh.clamp(min=0))
        q = 1 / (1 + torch.exp(bh))
        slope = -BETA * ((1 - SMOOTHING) * q - SMOOTHING * (1 - q)) / P
        both = torch.stack([slope, -slope], 1).reshape(-1) / count
        grad = _row_grad(e, total, at, both[s["sequence"]] * active.float(), s["logits"].dtype)
        return {"seq_logp": seq, "pair_loss": pair, "margin": bh, "loss": pair.sum().reshape(1) / P, "dlogits": grad}
    if op == "keep":
        x = s["x"].float()
        rows, cols = x.shape
        wide = torch.zeros((rows, (cols + 31) // 32 * 32), device=x.device)
        wide[:, :cols] = x
        blocks = wide.view(rows, -1, 32)
        step = torch.exp2(_exponent(blocks.abs().amax(2)))[:, :, None]
        restored = (torch.round(blocks / step) * step).view(rows, -1)[:, :cols].to(s["x"].dtype)
        return {"restored": restored, "value": None if case["act"] == "none" else _act(x, case["act"]).to(s["x"].dtype)}
    x = _restore(s["codes"], s["scales"], case["cols"])
    if op == "act_backward":
        return (s["dy"].float() * _slope(x, case["act"])).to(s["dy"].dtype)
    return (s["dy"].float().t() @ x).to(s["dw"].dtype)


# --------------------------------------------------------------------------
# The definitions in 64 bits
# --------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("policy", "logprobs", "preference"):
        return _exact_loss(case, s)
    if op == "keep":
        x = s["x"].double()
        rows, cols = x.shape
        restored = torch.empty_like(x)
        for a in range(0, cols, 32):
            part = x[:, a:a + 32]
            m, k = torch.frexp(part.abs().amax(1))              # largest = m 2^k, 1/2 <= m < 1
            e = torch.where(m * 128 < 127.5, k - 7, k - 6)
            e = torch.where(m == 0, torch.full_like(e, -126), e).clamp(min=-126)
            size = torch.ldexp(torch.ones_like(m), e)[:, None]
            restored[:, a:a + 32] = torch.round(part / size) * size
        return {"restored": restored, "value": None if case["act"] == "none" else _exact_act(x, case["act"])}
    x = torch.empty((case["rows"], case["cols"]), dtype=torch.float64, device="cuda")
    for a in range(0, case["cols"], 32):
        size = torch.ldexp(torch.ones((), dtype=torch.float64, device="cuda"), s["scales"][a // 128, :case["rows"], a // 32 % 4].int() - 127)
        b = min(case["cols"], a + 32)
        x[:, a:b] = s["codes"][:, a:b].double() * size[:, None]
    if op == "act_backward":
        x.requires_grad_(True)
        _exact_act(x, case["act"]).backward(s["dy"].double())
        return x.grad
    return torch.einsum("to,tc->oc", s["dy"].double(), x)


def _exact_act(x, act):
    if act == "gelu_tanh":
        return torch.nn.functional.gelu(x, approximate="tanh")
    if act == "gelu_erf":
        return torch.nn.functional.gelu(x)
    return torch.nn.functional.silu(x) if act == "silu" else x


def _exact_loss(case, s):
    rows, vocab = s["logits"].shape
    labels = s["labels"]
    step = max(1, (1 << 28) // vocab)
    at = labels.clamp(min=0)
    logp = torch.empty(rows, dtype=torch.float64, device="cuda")
    lse = torch.empty_like(logp)
    for a in range(0, rows, step):
        z = torch.log_softmax(s["logits"][a:a + step].double(), 1).gather(1, at[a:a + step, None])[:, 0]
        logp[a:a + step] = z
        lse[a:a + step] = s["logits"][a:a + step].gather(1, at[a:a + step, None])[:, 0].double() - z
    off = labels < 0
    logp[off], lse[off] = 0.0, 0.0
    if case["op"] == "logprobs":
        return logp, lse
    lp = logp.clone().requires_grad_(True)
    if case["op"] == "policy":
        w, a = s["weights"].double(), s["advantages"].double()
        r = torch.exp(lp - s["old"].double())
        u, c = r * a, r.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * a
        gain = torch.minimum(u, c)
        d = s["ref"].double() - lp if case["ref"] else torch.zeros_like(lp)
        kl = torch.exp(d) - d - 1
        token = torch.where(off, torch.zeros_like(lp), -gain + (KL if case["ref"] else 0.0) * kl)
        total = (w * token).sum()
        out = {"logp": logp, "token_loss": token.detach(),
               "sums": torch.stack([total, -(w * gain).sum(), (w * kl).sum(), (w * (u > c)).sum()]).detach()}
        if not case["grad"]:
            return {**out, "dlogits": None}
    else:
        n = s["offsets"].tolist()
        seq = torch.stack([lp[a:b].sum() / (max(1, int((~off[a:b]).sum())) if case["average"] else 1) for a, b in zip(n, n[1:])])
        h = seq[0::2] - seq[1::2]
        if case["ref"]:
            h = h - (s["ref"][0::2].double() - s["ref"][1::2].double())
        ls = torch.nn.functional.logsigmoid
        pair = -(1 - SMOOTHING) * ls(BETA * h) - SMOOTHING * ls(-BETA * h)
        total = pair.sum() / case["pairs"]
        out = {"seq_logp": seq.detach(), "pair_loss": pair.detach(), "margin": (BETA * h).detach(), "loss": total.detach().reshape(1)}
    total.backward()
    coef = torch.where(off, torch.zeros_like(lp.grad), lp.grad)
    # The gradient is kept in 32 bits: far finer than what it is compared with, and half the memory of 64.
    grad = torch.empty((rows, vocab), dtype=torch.float64 if rows * vocab <= 1 << 28 else torch.float32, device="cuda")
    for a in range(0, rows, step):
        p = torch.softmax(s["logits"][a:a + step].double(), 1)
        g = -coef[a:a + step, None] * p
        g.scatter_add_(1, at[a:a + step, None], coef[a:a + step, None])
        grad[a:a + step] = g
    return {**out, "dlogits": grad}
