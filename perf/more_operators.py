"""What is measured of the operators of a worker's distillation step: a teacher's
log-probabilities with entropy and top alternatives, and their backward pass; the
distillation loss from such a record with its gradient; and the root-mean-square
norm of a residual stream, its output kept in 8 bits, with its backward pass.

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
EPS = 1e-5


def listed():
    return [
        # A teacher's record of a batch of 4096 tokens, a third of them prompt: 64 alternatives each.
        dict(name="alternatives 4096 tokens", op="alternatives", rows=4096, vocab=GPT2_VOCAB, dtype=BF16, k=64, temperature=1.0, masked=0.3),
        # The answer of a server to one token: its log-probability, entropy and 20 alternatives.
        dict(name="alternatives 1 token", op="alternatives", rows=1, vocab=GPT2_VOCAB, dtype=BF16, k=20, temperature=1.0, masked=0.0),
        # A short record at a raised temperature, logits kept in fp32, a vocabulary of odd size.
        dict(name="alternatives 300 tokens fp32", op="alternatives", rows=300, vocab=32001, dtype=F32, k=8, temperature=2.0, masked=0.1),
        # The gradient of a policy objective with an entropy bonus, one micro-batch of 8 sequences.
        dict(name="alternatives backward 8192 tokens", op="alternatives_backward", rows=8192, vocab=GPT2_VOCAB, dtype=BF16, k=0, temperature=1.0, masked=0.35),
        # The gradient through recorded alternatives too, for the last short completion of an epoch.
        dict(name="alternatives backward 37 tokens fp32", op="alternatives_backward", rows=37, vocab=32001, dtype=F32, k=20, temperature=1.0, masked=0.2),
        # One micro-batch of distillation from 64 recorded log-probabilities a token and what they leave.
        dict(name="distillation 8x1024 tokens", op="distillation", rows=8192, vocab=GPT2_VOCAB, dtype=BF16, k=64, temperature=1.0, rest=True, label=0.0, masked=0.35),
        # Softened targets (temperature 2) from 32 logits, mixed with the labels' cross-entropy.
        dict(name="distillation 2048 tokens labels", op="distillation", rows=2048, vocab=GPT2_VOCAB, dtype=BF16, k=32, temperature=2.0, rest=False, label=0.3, masked=0.35),
        # The last, short completion, logits kept in fp32.
        dict(name="distillation 37 tokens fp32", op="distillation", rows=37, vocab=32001, dtype=F32, k=16, temperature=1.0, rest=True, label=0.5, masked=0.2),
        # The norm in front of an MLP over 16 sequences of 1024 tokens, for training.
        dict(name="norm 16384x4096", op="norm", rows=16384, cols=4096, dtype=BF16, residual=True, keep=True),
        # The same for one token, as a server runs it.
        dict(name="norm 1x4096", op="norm", rows=1, cols=4096, dtype=BF16, residual=True, keep=False),
        # Its backward pass over the 16 sequences.
        dict(name="norm backward 16384x4096", op="norm_backward", rows=16384, cols=4096, dtype=BF16, residual=True, keep=False),
        # An odd width in fp32, the stream kept in 8 bits.
        dict(name="norm backward 300x1001 fp32", op="norm_backward", rows=300, cols=1001, dtype=F32, residual=False, keep=True),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["alternatives", "alternatives_backward", "distillation", "norm", "norm_backward"])
    dtype = rng.choice([BF16, BF16, BF16, F32])
    if op in ("norm", "norm_backward"):
        cols = _spread(rng, 64, 8192)
        if rng.random() < 0.7:
            cols = cols // 8 * 8
        rows = min(_spread(rng, 1, 16384), 16384 * 4096 * 2 // (cols * SIZE[dtype]))
        return dict(op=op, rows=rows, cols=cols, dtype=dtype, residual=rng.random() < 0.7, keep=rng.random() < 0.6)
    vocab = _spread(rng, 2000, 131072)
    if rng.random() < 0.5:
        vocab = vocab // 64 * 64
    most = (4096 if op == "alternatives" else 8192) * GPT2_VOCAB * 2 // (vocab * SIZE[dtype])
    case = dict(op=op, rows=min(_spread(rng, 1, 16384), most), vocab=vocab, dtype=dtype, k=_spread(rng, 1, 128),
                temperature=rng.choice([1.0, 1.0, 2.0, round(rng.uniform(0.5, 4.0), 2)]), masked=round(rng.uniform(0.0, 0.6), 2))
    if op == "alternatives_backward" and rng.random() < 0.5:
        case["k"] = 0
    if op == "distillation":
        case.update(rest=rng.random() < 0.5, label=rng.choice([0.0, round(rng.uniform(0.1, 0.9), 2)]))
        if case["label"] and case["temperature"] != 1.0:
            case["rows"] = max(1, case["rows"] // 2)
    return case


def work(case):
    s, op, rows = SIZE[case["dtype"]], case["op"], case["rows"]
    if op == "norm":
        n = rows * case["cols"]
        kept = n + n / 32 if case["keep"] else 0                # codes and scales, written and read again; values of 2 bytes
        return {"bytes": n * s * (4 if case["residual"] else 2) + 2 * kept + (2 * n if case["keep"] else 0) + 4 * rows, "flops": 8 * n}
    if op == "norm_backward":
        n = rows * case["cols"]
        return {"bytes": n * s * (3 if case["residual"] else 2) + (n + n / 32 if case["keep"] else n * s) + 4 * rows, "flops": 10 * n}
    read = rows - _masked_rows(case)                            # masked rows' logits are not needed
    write = 0 if op == "alternatives" else rows
    passes = {"alternatives": 5, "alternatives_backward": 5, "distillation": 8 if _two_softmaxes(case) else 4}[op]
    return {"bytes": (read + write) * case["vocab"] * s + rows * (24 + 8 * case["k"]), "flops": passes * read * case["vocab"]}


def _two_softmaxes(case):
    return case.get("label", 0.0) != 0.0 and case["temperature"] != 1.0


# --------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------
def _masked_rows(case):
    return int(case["rows"] * case["masked"])


def _logits(gen, rows, vocab, dtype):
    """Logits of a language model and labels: the label's log-probability is about -exponential(1.3)."""
    x = torch.empty((rows, vocab), dtype=TORCH_TYPE[dtype], device="cuda")
    labels = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    for a, b in _parts(rows, vocab, 26):
        z = torch.empty((b - a, vocab), device="cuda").normal_(0.0, 2.0, generator=gen)
        want = torch.empty(b - a, device="cuda").exponential_(1 / 1.3, generator=gen).clamp_(0.02, 12.0)
        rest = torch.logsumexp(z, 1)
        z.scatter_(1, labels[a:b, None], (rest - torch.log(torch.expm1(want)))[:, None])
        x[a:b] = z
    return x, labels


def _parts(rows, vocab, log_elements):
    step = max(1, (1 << log_elements) // vocab)
    return [(a, min(rows, a + step)) for a in range(0, rows, step)]


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
    s = {"case": case}
    rows = case["rows"]
    if case["op"] in ("norm", "norm_backward"):
        return _prepare_norm(case, gen, s)
    vocab, k, T = case["vocab"], case["k"], case["temperature"]
    x, labels = _logits(gen, rows, vocab, case["dtype"])
    drop = torch.randperm(rows, generator=gen, device="cuda")[:_masked_rows(case)]
    labels[drop] = -100
    s.update(logits=x, labels=labels)
    randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    if case["op"] == "alternatives":
        s.update(ids=torch.empty((rows, k), dtype=torch.int32, device="cuda"), top=torch.empty((rows, k), device="cuda"),
                 logp=torch.empty(rows, device="cuda"), lse=torch.empty(rows, device="cuda"), entropy=torch.empty(rows, device="cuda"))
        return s
    s["dlogits"] = torch.empty_like(x)
    active = labels >= 0
    n = max(1, rows - _masked_rows(case))
    if case["op"] == "alternatives_backward":
        # What the forward pass gave, and the gradients of its results.
        lse, entropy = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        ids = torch.empty((rows, k), dtype=torch.int32, device="cuda")
        for a, b in _parts(rows, vocab, 26):
            z = x[a:b].float() / T
            lse[a:b] = torch.logsumexp(z, 1)
            p = torch.softmax(z, 1)
            entropy[a:b] = lse[a:b] - (p * z).sum(1)
            ids[a:b] = torch.topk(z, k, 1)[1].int()
        lse[~active], entropy[~active], ids[~active] = -math.inf, 0.0, -1
        s.update(lse=lse, entropy=entropy, ids=ids if k else None, d_logp=randn(rows) / n, d_entropy=0.01 * torch.rand(rows, generator=gen, device="cuda") / n,
                 d_top=randn(rows, k) / (n * k) if k else None)
        return s
    # A teacher that differs from the student by noise of 0.7 a logit.
    ids = torch.empty((rows, k), dtype=torch.int32, device="cuda")
    values = torch.empty((rows, k), device="cuda")
    for a, b in _parts(rows, vocab, 26):
        z = x[a:b].float() + 0.7 * torch.empty((b - a, vocab), device="cuda").normal_(generator=gen)
        if case["rest"]:
            z = torch.log_softmax(z / T, 1)
        top = torch.topk(z, k, 1)
        values[a:b], ids[a:b] = top.values, top.indices.int()
    ids[drop], values[drop] = -1, -math.inf
    s.update(ids=ids, values=values, weights=active.float() / n, token_loss=torch.empty(rows, device="cuda"), sums=torch.empty(4, device="cuda"),
             workspace=torch.empty((1 << 20) + 64 * rows, dtype=torch.uint8, device="cuda"))
    return s


def _prepare_norm(case, gen, s):
    rows, cols, t = case["rows"], case["cols"], TORCH_TYPE[case["dtype"]]
    randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    # A residual stream: Gaussian, with a few columns that are ten times as large.
    wide = 1 + 9 * (torch.rand(cols, generator=gen, device="cuda") < 0.01).float()
    x = (randn(rows, cols) * wide).to(t)
    s.update(gain=(1 + 0.1 * randn(cols)).to(t), rstd=torch.empty(rows, device="cuda"))
    if case["op"] == "norm":
        s.update(x=x, residual=(randn(rows, cols) * wide).to(t) if case["residual"] else None, y=torch.empty_like(x),
                 total=torch.empty_like(x) if case["residual"] else None)
        if case["keep"]:
            s.update(codes=torch.empty((rows, (cols + 15) // 16 * 16), dtype=torch.int8, device="cuda"),
                     scales=torch.empty(((cols + 127) // 128, (rows + 63) // 64 * 64, 4), dtype=torch.uint8, device="cuda"),
                     restored=torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda"))
        return s
    s["rstd"] = torch.rsqrt(x.double().square().mean(1) + EPS).float()
    s.update(dy=(1e-3 * randn(rows, cols)).to(t), d_total=(1e-3 * randn(rows, cols)).to(t) if case["residual"] else None,
             dx=torch.empty_like(x), dgain=torch.empty(cols, dtype=t, device="cuda"),
             workspace=torch.empty((1 << 20) + 4096 * 4 * cols, dtype=torch.uint8, device="cuda"))
    if case["keep"]:
        s["codes"], s["scales"] = _kept(x)
    else:
        s["x"] = x
    return s


# --------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------
def run(s):
    return (_own if own else _plain)(s["case"], s)


def _own(case, s):
    from paper_2512_09685_b200 import binding as star
    op = case["op"]
    if op == "alternatives":
        star.star_token_alternatives(s["logits"], s["ids"], s["top"], labels=s["labels"], logp=s["logp"], lse=s["lse"], entropy=s["entropy"],
                                     temperature=case["temperature"])
        return {"ids": s["ids"], "top": s["top"], "logp": s["logp"], "lse": s["lse"], "entropy": s["entropy"]}
    if op == "alternatives_backward":
        star.star_token_alternatives_backward(s["dlogits"], s["logits"], s["lse"], labels=s["labels"], d_logp=s["d_logp"], entropy=s["entropy"],
                                              d_entropy=s["d_entropy"], top_ids=s["ids"], d_top_logp=s["d_top"], temperature=case["temperature"])
        return s["dlogits"]
    if op == "distillation":
        star.star_distillation_loss(s["logits"], s["ids"], s["values"], s["token_loss"], s["sums"], s["workspace"], dlogits=s["dlogits"],
                                    labels=s["labels"], weights=s["weights"], temperature=case["temperature"],
                                    teacher_temperature=1.0 if case["rest"] else case["temperature"], rest=case["rest"],
                                    soft_coef=1.0 - case["label"], label_coef=case["label"])
        return {"token_loss": s["token_loss"], "sums": s["sums"], "dlogits": s["dlogits"]}
    if op == "norm":
        star.star_rms_norm(s["y"], s["x"], s["gain"], residual=s["residual"], total=s["total"], rstd=s["rstd"],
                           codes=s.get("codes"), scales=s.get("scales"), eps=EPS)
        if case["keep"]:
            star.star_checkpoint_unpack(s["restored"], s["codes"], s["scales"])
        return {"y": s["y"], "total": s["total"], "rstd": s["rstd"], "restored": s.get("restored")}
    star.star_rms_norm_backward(s["dx"], s["dgain"], s["dy"], s["gain"], s["rstd"], s["workspace"], total=s.get("x"), codes=s.get("codes"),
                                scales=s.get("scales"), d_total=s["d_total"])
    return {"dx": s["dx"], "dgain": s["dgain"]}


def _softmax_parts(x, temperature):
    """Logits over the temperature, their largest, exponentials and the exponentials' sum."""
    z = x.float() / temperature
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    return z, top, e, e.sum(1, keepdim=True)


def _plain(case, s):
    op = case["op"]
    if op == "norm":
        total = (s["x"].float() + s["residual"].float()).to(s["x"].dtype) if case["residual"] else None
        x = (s["x"] if total is None else total).float()
        rstd = 1 / torch.sqrt((x * x).mean(1) + EPS)
        y = (x * rstd[:, None] * s["gain"].float()).to(s["x"].dtype)
        return {"y": y, "total": total, "rstd": rstd, "restored": _through_8_bits(y).to(torch.bfloat16) if case["keep"] else None}
    if op == "norm_backward":
        x = _restore(s["codes"], s["scales"], case["cols"]) if case["keep"] else s["x"].float()
        dy = s["dy"].float()
        n, g = x * s["rstd"][:, None], dy * s["gain"].float()
        dx = s["rstd"][:, None] * (g - n * (g * n).mean(1, keepdim=True))
        if case["residual"]:
            dx = dx + s["d_total"].float()
        return {"dx": dx.to(s["dy"].dtype), "dgain": (dy * n).sum(0).to(s["dgain"].dtype)}
    active = s["labels"] >= 0
    at = s["labels"].clamp(min=0)[:, None]
    off = torch.zeros(active.shape, device="cuda")
    if op == "alternatives":
        z, top, e, total = _softmax_parts(s["logits"], case["temperature"])
        low = z - top
        logp = (low.gather(1, at) - torch.log(total))[:, 0]
        lse = (top + torch.log(total))[:, 0]
        entropy = (torch.log(total) - (e * low).sum(1, keepdim=True) / total)[:, 0]
        # The largest logits, equal ones by the lowest index: the logit's order in the high bits of one number, the index in the low ones.
        bits = (s["logits"].float() + 0.0).view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7fffffff, bits).to(torch.int64)
        key = (order << 32) + (0x7fffffff - torch.arange(case["vocab"], device="cuda"))
        ids = 0x7fffffff - (torch.topk(key, case["k"], 1, sorted=True)[0] & 0xffffffff)
        best = low.gather(1, ids) - torch.log(total)
        return {"ids": torch.where(active[:, None], ids.int(), -1), "top": torch.where(active[:, None], best, -math.inf), "logp": torch.where(active, logp, off),
                "lse": torch.where(active, lse, -math.inf), "entropy": torch.where(active, entropy, off)}
    if op == "alternatives_backward":
        u = s["logits"].float() / case["temperature"] - torch.where(active, s["lse"], off)[:, None]
        h = s["d_entropy"]
        each = s["d_logp"] if not case["k"] else s["d_logp"] + s["d_top"].sum(1)
        g = -torch.exp(u) * (each[:, None] + h[:, None] * (u + s["entropy"][:, None]))
        g.scatter_add_(1, at, s["d_logp"][:, None])
        if case["k"]:
            g.scatter_add_(1, s["ids"].clamp(min=0).long(), s["d_top"])
        return torch.where(active[:, None], g / case["temperature"], 0.0).to(s["logits"].dtype)
    # Distillation.  What is made of the few listed entries of a row is held in 64 bits, the vocabulary in 32.
    T, soft, hard = case["temperature"], 1.0 - case["label"], case["label"]
    ids, present = s["ids"].clamp(min=0).long(), s["ids"] >= 0
    z, top, e, total = _softmax_parts(s["logits"], T)
    log_total = torch.log(total.double())
    logp = z.gather(1, ids).double() - top.double() - log_total
    ce = torch.where(active, (log_total + top.double() - z.gather(1, at).double())[:, 0], 0.0)
    u = s["values"].double() / (1.0 if case["rest"] else T)
    if not case["rest"]:
        u = u - torch.logsumexp(torch.where(active[:, None], u, 0.0), 1, keepdim=True)
    q = torch.where(present, torch.exp(u), 0.0)
    kl = (q * torch.where(q > 0, u - logp, 0.0)).sum(1)
    mass = q.sum(1, keepdim=True)
    q0 = (1 - mass).clamp(min=0) if case["rest"] else torch.zeros_like(mass)
    rest = e.scatter(1, ids, 0.0).sum(1, keepdim=True)
    if case["rest"]:
        kl = kl + torch.where(q0 > 0, q0 * (torch.log(q0) - torch.log(rest.double()) + log_total), 0.0)[:, 0]
    w = torch.where(active, s["weights"], off)
    scale = (mass + q0).float() / total
    g = e * (scale - q0.float() / rest)
    g.scatter_(1, ids, e.gather(1, ids) * scale - q.float())
    g *= soft / T
    if hard:
        p = e / total
        if T != 1.0:
            z1, top1, p, total1 = _softmax_parts(s["logits"], 1.0)
            ce = torch.where(active, (torch.log(total1.double()) + top1.double() - z1.gather(1, at).double())[:, 0], 0.0)
            p = p / total1
        g += hard * p
        g.scatter_add_(1, at, torch.full_like(w, -hard)[:, None])
    kl = torch.where(active, kl, 0.0)
    loss = soft * kl + hard * ce
    w64 = w.double()
    sums = torch.stack([(w64 * loss).sum(), (w64 * kl).sum(), (w64 * ce).sum() if hard else w64.sum() * 0.0, w64.sum()])
    return {"token_loss": loss.float(), "sums": sums.float(), "dlogits": torch.where(active[:, None], g * w[:, None], 0.0).to(s["logits"].dtype)}


def _through_8_bits(y):
    rows, cols = y.shape
    wide = torch.zeros((rows, (cols + 31) // 32 * 32), device=y.device)
    wide[:, :cols] = y.float()
    blocks = wide.view(rows, -1, 32)
    step = torch.exp2(_exponent(blocks.abs().amax(2)))[:, :, None]
    return (torch.round(blocks / step) * step).view(rows, -1)[:, :cols]


def _restore(codes, scales, cols):
    rows = codes.shape[0]
    e = scales[:, :rows].transpose(0, 1).reshape(rows, -1).float() - 127
    return codes[:, :cols].float() * torch.exp2(e).repeat_interleave(32, 1)[:, :cols]


# --------------------------------------------------------------------------
# The definitions in 64 bits
# --------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "norm_backward": _exact_norm_backward, "alternatives": _exact_alternatives,
            "alternatives_backward": _exact_alternatives_backward, "distillation": _exact_distillation}[case["op"]](case, s)


def _exact_norm(case, s):
    x, total = s["x"].double(), None
    if case["residual"]:
        x = x + s["residual"].double()
        total = x
        x = x.to(s["x"].dtype).double()                         # the norm is of the stream as it is kept
    size = torch.linalg.vector_norm(x, dim=1).square() / case["cols"]
    rstd = (size + EPS).pow(-0.5)
    y = torch.einsum("tc,t,c->tc", x, rstd, s["gain"].double())
    restored = None
    if case["keep"]:
        kept = y.to(s["x"].dtype).double()
        restored = torch.empty_like(kept)
        for a in range(0, case["cols"], 32):
            part = kept[:, a:a + 32]
            m, k = torch.frexp(part.abs().amax(1))              # largest = m 2^k, 1/2 <= m < 1
            e = torch.where(m * 128 < 127.5, k - 7, k - 6)
            e = torch.where(m == 0, torch.full_like(e, -126), e).clamp(min=-126)
            unit = torch.ldexp(torch.ones_like(m), e)[:, None]
            restored[:, a:a + 32] = torch.round(part / unit) * unit
    return {"y": y, "total": total, "rstd": rstd, "restored": restored}


def _exact_norm_backward(case, s):
    if case["keep"]:
        x = torch.empty((case["rows"], case["cols"]), dtype=torch.float64, device="cuda")
        for a in range(0, case["cols"], 32):
            unit = torch.ldexp(torch.ones((), dtype=torch.float64, device="cuda"), s["scales"][a // 128, :case["rows"], a // 32 % 4].int() - 127)
            b = min(case["cols"], a + 32)
            x[:, a:b] = s["codes"][:, a:b].double() * unit[:, None]
    else:
        x = s["x"].double()
    dy, r, gain = s["dy"].double(), s["rstd"].double(), s["gain"].double()
    inner = torch.einsum("tc,tc,c->t", dy, x, gain) * r ** 3 / case["cols"]
    dx = torch.einsum("tc,t,c->tc", dy, r, gain) - x * inner[:, None]
    if case["residual"]:
        dx = dx + s["d_total"].double()
    return {"dx": dx, "dgain": torch.einsum("tc,tc,t->c", dy, x, r)}


def _exact_alternatives(case, s):
    rows, vocab, k = case["rows"], case["vocab"], case["k"]
    off = s["labels"] < 0
    at = s["labels"].clamp(min=0)
    new = lambda *shape: torch.empty(shape, dtype=torch.float64, device="cuda")  # noqa: E731
    out = {"ids": torch.empty((rows, k), dtype=torch.int32, device="cuda"), "top": new(rows, k), "logp": new(rows), "lse": new(rows), "entropy": new(rows)}
    for a, b in _parts(rows, vocab, 26):
        z = s["logits"][a:b].double() / case["temperature"]
        every = torch.log_softmax(z, 1)
        out["lse"][a:b] = torch.logsumexp(z, 1)
        out["logp"][a:b] = every.gather(1, at[a:b, None])[:, 0]
        out["entropy"][a:b] = torch.special.entr(every.exp()).sum(1)
        first = torch.sort(s["logits"][a:b].float(), dim=1, descending=True, stable=True)[1][:, :k]
        out["ids"][a:b] = first.int()
        out["top"][a:b] = every.gather(1, first)
    out["ids"][off], out["top"][off], out["logp"][off], out["lse"][off], out["entropy"][off] = -1, -math.inf, 0.0, -math.inf, 0.0
    return out


def _wide(rows, vocab):
    """A gradient kept in 32 bits where it is large: far finer than what it is compared with, and half the memory."""
    return torch.zeros((rows, vocab), dtype=torch.float64 if rows * vocab <= 1 << 28 else torch.float32, device="cuda")


def _exact_alternatives_backward(case, s):
    rows, vocab = case["rows"], case["vocab"]
    grad = _wide(rows, vocab)
    for a, b in _parts(rows, vocab, 27):
        on = torch.nonzero(s["labels"][a:b] >= 0)[:, 0] + a
        u = s["logits"][on].double() / case["temperature"] - s["lse"][on].double()[:, None]
        hot = torch.zeros_like(u)
        hot[torch.arange(len(on), device="cuda"), s["labels"][on]] = s["d_logp"][on].double()
        if case["k"]:
            hot.scatter_add_(1, s["ids"][on].long(), s["d_top"][on].double())
        p = u.exp()
        h = s["d_entropy"][on].double()[:, None]
        g = hot - p * hot.sum(1, keepdim=True) - h * p * (u + s["entropy"][on].double()[:, None])
        grad[on] = (g / case["temperature"]).to(grad.dtype)
    return grad


def _exact_distillation(case, s):
    rows, vocab, T, hard = case["rows"], case["vocab"], case["temperature"], case["label"]
    grad = _wide(rows, vocab)
    kl, ce = torch.zeros(rows, dtype=torch.float64, device="cuda"), torch.zeros(rows, dtype=torch.float64, device="cuda")
    for a, b in _parts(rows, vocab, 26):
        on = torch.nonzero(s["labels"][a:b] >= 0)[:, 0] + a
        if not len(on):
            continue
        x = s["logits"][on].double().requires_grad_(True)
        every = torch.log_softmax(x / T, 1)
        ids = s["ids"][on].long()
        logq = s["values"][on].double()
        if not case["rest"]:
            logq = torch.log_softmax(logq / T, 1)
        q = logq.exp()
        part = (q * (logq - every.gather(1, ids))).sum(1)
        if case["rest"]:
            q0 = (1 - q.sum(1)).clamp(min=0)
            apart = torch.logsumexp(every.scatter(1, ids, -math.inf), 1)
            part = part + torch.where(q0 > 0, q0 * (q0.log() - apart), torch.zeros_like(q0))
        loss = (1 - hard) * part
        if hard:
            cross = torch.nn.functional.cross_entropy(x, s["labels"][on], reduction="none")
            loss = loss + hard * cross
            ce[on] = cross.detach()
        (loss * s["weights"][on].double()).sum().backward()
        kl[on] = part.detach()
        grad[on] = x.grad.to(grad.dtype)
    w = torch.where(s["labels"] >= 0, s["weights"], torch.zeros_like(s["weights"])).double()
    token = (1 - hard) * kl + hard * ce
    return {"token_loss": token, "sums": torch.stack([(w * token).sum(), (w * kl).sum(), (w * ce).sum(), w.sum()]), "dlogits": grad}
