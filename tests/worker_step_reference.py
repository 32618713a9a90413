"""The operators of a worker's step in binary64, written from their formulas
(plain torch, any device); what the GPU tests compare the kernels with."""
import math

import torch

ACTS = ("none", "gelu_tanh", "gelu_erf", "silu")


def rows(logits, labels, weights=None, temperature=1.0):
    """(logp, lse, p, active) of every row; inactive rows have logp = lse = 0."""
    T, V = logits.shape
    x = logits.double()
    z = x / temperature
    active = (labels >= 0) & (labels < V)
    if weights is not None:
        active = active & (weights != 0)
    x = torch.where(active[:, None], x, torch.zeros_like(x))          # inactive rows are not read
    z = torch.where(active[:, None], z, torch.zeros_like(z))
    if V:
        active = active & ~(z == -math.inf).all(1)
    z = torch.where(active[:, None], z, torch.zeros_like(z))
    top = z.amax(1, keepdim=True) if V else z.new_zeros(T, 1)
    e = torch.exp(z - top)
    s = e.sum(1, keepdim=True)
    lse = (top + torch.log(s))[:, 0] if V else z.new_zeros(T)
    at = torch.where(active, labels, torch.zeros_like(labels))
    logp = ((z.gather(1, at[:, None]) - top) - torch.log(s))[:, 0] if V else z.new_zeros(T)     # exact also where top is huge
    off = torch.zeros_like(logp)
    return torch.where(active, logp, off), torch.where(active, lse, off), e / s, active


def gradient(p, labels, active, coef):
    """coef * (onehot - p), 0 for inactive rows."""
    hot = torch.zeros_like(p)
    at = torch.where(active, labels, torch.zeros_like(labels))
    if p.shape[1]:
        hot.scatter_(1, at[:, None], 1.0)
    return torch.where(active[:, None], coef[:, None] * (hot - p), torch.zeros_like(p))


def policy(logits, labels, advantages, weights=None, old=None, ref=None, clip_low=0.2, clip_high=0.2, kl_coef=0.0,
           temperature=1.0):
    lp, _, p, active = rows(logits, labels, weights, temperature)
    w = torch.ones_like(lp) if weights is None else weights.double()
    A = advantages.double()
    r = torch.exp(lp - old.double()) if old is not None else torch.ones_like(lp)
    u = r * A
    c = r.clamp(1 - clip_low, 1 + clip_high) * A
    gain = torch.where(u > c, c, u)
    slope = torch.where(u > c, torch.zeros_like(u), -u)
    kl = torch.zeros_like(lp)
    if ref is not None:
        d = ref.double() - lp
        kl = torch.expm1(d) - d
        slope = slope - kl_coef * torch.expm1(d)
    off = torch.zeros_like(lp)
    loss = torch.where(active, -gain + kl_coef * kl, off)
    part = lambda x: torch.where(active, w * x, off).sum()  # noqa: E731
    sums = torch.stack([part(loss), part(-gain), part(kl), part((u > c).double())])
    return {"logp": lp, "token_loss": loss, "sums": sums, "dlogits": gradient(p, labels, active, w * slope / temperature),
            "active": active, "margin_to_clip": (u - c).abs()}


def preference(logits, labels, offsets, ref=None, beta=0.1, smoothing=0.0, average=False, scale=1.0, temperature=1.0):
    lp, _, p, active = rows(logits, labels, None, temperature)
    T = logits.shape[0]
    n = [min(max(int(o), 0), T) for o in offsets]
    seqs = list(zip(n, n[1:]))
    L, counts = [], []
    for a, b in seqs:
        k = int(active[a:b].sum()) if b > a else 0
        counts.append(max(k, 1) if average else 1)
        L.append(lp[a:b].sum() / counts[-1] if b > a else lp.new_zeros(()))
    seq = torch.stack(L) if L else lp.new_zeros(0)
    h = seq[0::2] - seq[1::2]
    if ref is not None:
        h = h - (ref.double()[0::2] - ref.double()[1::2])
    bh = beta * h
    soft = lambda x: torch.log1p(torch.exp(-x.abs())) + torch.clamp(-x, min=0)  # noqa: E731
    pair = (1 - smoothing) * soft(bh) + (smoothing * soft(-bh) if smoothing else 0.0)
    slope = -beta * ((1 - smoothing) * torch.sigmoid(-bh) - smoothing * torch.sigmoid(bh))
    coef = torch.zeros_like(lp)
    for s, (a, b) in enumerate(seqs):
        if b > a:
            coef[a:b] = (-1 if s % 2 else 1) * slope[s // 2] * scale / temperature / counts[s]
    return {"seq_logp": seq, "pair_loss": pair, "margin": bh, "loss": (scale * pair.sum()).reshape(1),
            "dlogits": gradient(p, labels, active, coef)}


def act(x, name):
    if name == "gelu_tanh":
        return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))
    if name == "gelu_erf":
        return 0.5 * x * torch.erfc(-x / math.sqrt(2))
    if name == "silu":
        return x * torch.sigmoid(x)
    return x


def act_slope(x, name):
    if name == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * (x + 0.044715 * x ** 3))
        return 0.5 * (1 + t) + 0.5 * x * (1 - t * t) * k * (1 + 3 * 0.044715 * x * x)
    if name == "gelu_erf":
        return 0.5 * torch.erfc(-x / math.sqrt(2)) + x * torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)
    if name == "silu":
        q = torch.sigmoid(x)
        return q * (1 + x * (1 - q))
    return torch.ones_like(x)


def power_of_two(e):
    """2^e in binary64 from its bits (a power function need not be exact on every device)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def kept(x):
    """(codes [rows, cols], scale bytes [rows, blocks], values [rows, cols] in binary64), block by block."""
    T, C = x.shape
    blocks = (C + 31) // 32
    codes = torch.zeros((T, C), dtype=torch.int8, device=x.device)
    scale = torch.zeros((T, blocks), dtype=torch.int64, device=x.device)
    values = torch.zeros((T, C), dtype=torch.float64, device=x.device)
    for b in range(blocks):
        part = x[:, 32 * b: 32 * b + 32].double()
        largest = part.abs().amax(1)
        bad = ~torch.isfinite(part).all(1) | (largest >= 127.5 * 2.0 ** 104)
        e = torch.full((T,), -126, dtype=torch.int64, device=x.device)
        for _ in range(240):                              # the smallest exponent that fits, by its definition
            too_small = ~bad & (torch.round(torch.where(bad, torch.zeros_like(largest), largest) * power_of_two(-e)) > 127)
            if not bool(too_small.any()):
                break
            e = e + too_small.long()
        step = power_of_two(e)
        q = torch.round(torch.where(bad[:, None], torch.zeros_like(part), part) / step[:, None])
        codes[:, 32 * b: 32 * b + 32] = q.to(torch.int8)
        scale[:, b] = torch.where(bad, torch.full_like(e, 255), e + 127)
        values[:, 32 * b: 32 * b + 32] = torch.where(bad[:, None], torch.full_like(part, math.nan), q * step[:, None])
    return codes, scale, values


def scale_bytes(scales, T, C):
    """[rows, blocks] from the buffer's layout."""
    blocks = (C + 31) // 32
    tall = (T + 63) // 64 * 64
    flat = scales.reshape(-1).long()
    t = torch.arange(T, device=scales.device)[:, None]
    b = torch.arange(blocks, device=scales.device)[None, :]
    return flat[((b // 4) * tall + t) * 4 + b % 4]


def rel(got, want):
    """|got - want| in the 2-norm over |want|; infinite where they are not finite in the same places."""
    got, want = got.double().reshape(-1), want.double().reshape(-1)
    assert got.shape == want.shape
    nan = torch.isnan(want)
    if not torch.equal(nan, torch.isnan(got)):
        return math.inf
    inf = torch.isinf(want)
    if not torch.equal(got[inf], want[inf]):
        return math.inf
    ok = ~(nan | inf)
    d, n = float(torch.linalg.vector_norm((got - want)[ok])), float(torch.linalg.vector_norm(want[ok]))
    return 0.0 if d == 0 else (d / n if n else math.inf)
