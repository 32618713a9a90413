"""A teacher's record, the distillation loss and the residual norm in binary64,
written from their formulas (plain torch, any device); what the tests compare the
kernels with, together with bounds on the kernels' rounding."""
import math

import torch

ULP = 2.0 ** -24                                       # half a step of binary32, relative


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def statistics(logits, labels=None, temperature=1.0):
    """(z, every log p, lse, entropy, active); inactive rows have lse -inf and entropy 0."""
    z = logits.double() / temperature
    rows, vocab = z.shape
    active = torch.ones(rows, dtype=torch.bool, device=z.device)
    if labels is not None:
        active = (labels >= 0) & (labels < vocab)
    z = torch.where(active[:, None], z, torch.full_like(z, -math.inf))            # inactive rows are not read
    active = active & ~(z == -math.inf).all(1)
    safe = torch.where(active[:, None], z, torch.zeros_like(z))
    top = safe.amax(1, keepdim=True)
    s = torch.exp(safe - top).sum(1, keepdim=True)
    every = (safe - top) - torch.log(s)                                           # exact also where top is huge
    p = torch.exp(every)
    entropy = -torch.where(p > 0, p * every, torch.zeros_like(p)).sum(1)
    lse = (top + torch.log(s))[:, 0]
    bad = torch.isnan(s[:, 0])
    entropy = torch.where(bad, torch.full_like(entropy, math.nan), entropy)
    off = torch.zeros_like(lse)
    return z, every, torch.where(active, lse, torch.full_like(lse, -math.inf)), torch.where(active, entropy, off), active


def alternatives(logits, k, labels=None, temperature=1.0):
    z, every, lse, entropy, active = statistics(logits, labels, temperature)
    rows, vocab = z.shape
    whole = active & torch.isfinite(lse)
    ids = torch.full((rows, k), -1, dtype=torch.int64, device=z.device)
    top = torch.full((rows, k), -math.inf, dtype=torch.float64, device=z.device)
    top[active & ~whole] = math.nan
    for t in torch.nonzero(whole)[:, 0].tolist():
        row = logits[t].double() + 0.0                 # -0 as 0
        order = torch.sort(row, descending=True, stable=True)[1][:k]
        order = order[row[order] > -math.inf]
        ids[t, :len(order)] = order
        top[t, :len(order)] = every[t, order]
    logp = torch.zeros_like(lse)
    if labels is not None:
        at = torch.where(active, labels, torch.zeros_like(labels))
        logp = torch.where(active, every.gather(1, at[:, None])[:, 0], logp)
    return {"ids": ids, "top": top, "logp": logp, "lse": lse, "entropy": entropy, "every": every, "active": active, "z": z}


def log_bound(x, every):
    """What a log-probability may be off: the sum's terms each by a few half steps and by one for every unit of their
    exponent, whose mean is below that of |log p|; the difference's own steps."""
    p = every.exp()
    mean = torch.where(p > 0, -p * every, torch.zeros_like(p)).sum(1, keepdim=True)
    return ULP * (32 + 8 * mean + 8 * x.abs().clamp(max=1e30))


def alternatives_backward(logits, lse, labels=None, d_logp=None, entropy=None, d_entropy=None, ids=None, d_top=None, temperature=1.0):
    """(gradient, bound on the kernel's rounding before the last one)."""
    rows, vocab = logits.shape
    active = lse != -math.inf
    if labels is not None:
        active = active & (labels >= 0) & (labels < vocab)
    x = torch.where(active[:, None], logits.double(), torch.zeros(1, dtype=torch.float64, device=logits.device))
    u = x / temperature - torch.where(active, lse.double(), torch.zeros_like(lse.double()))[:, None]
    p = torch.exp(u)
    hot = torch.zeros_like(p)
    size = torch.zeros_like(p)
    total = torch.zeros(rows, dtype=torch.float64, device=x.device)
    total_size = torch.zeros_like(total)
    if d_logp is not None:
        at = torch.where(active, labels, torch.zeros_like(labels))[:, None]
        hot.scatter_add_(1, at, d_logp.double()[:, None])
        size.scatter_add_(1, at, d_logp.double().abs()[:, None])
        total, total_size = total + d_logp.double(), total_size + d_logp.double().abs()
    if ids is not None:
        there = (ids >= 0) & (ids < vocab)
        g = torch.where(there, d_top.double(), torch.zeros(1, dtype=torch.float64, device=x.device))
        at = torch.where(there, ids, torch.zeros_like(ids)).long()
        hot.scatter_add_(1, at, g)
        size.scatter_add_(1, at, g.abs())
        total, total_size = total + g.sum(1), total_size + g.abs().sum(1)
    h = torch.zeros(rows, dtype=torch.float64, device=x.device) if d_entropy is None else d_entropy.double()
    H = torch.zeros_like(h) if entropy is None else entropy.double()
    pu = torch.where(p > 0, p * u, torch.zeros_like(p))
    grad = (hot - p * (total + h * H)[:, None] - h[:, None] * pu) / temperature
    depth = u.abs().clamp(max=200.0)
    bound = ULP * ((16 + 4 * depth) * (p * (total_size + h.abs() * H.abs())[:, None] + h.abs()[:, None] * pu.abs()) + 12 * size) / temperature + 1e-36
    off = torch.zeros_like(grad)
    return torch.where(active[:, None], grad, off), torch.where(active[:, None], bound, off)


def distillation(logits, ids, values, labels=None, weights=None, temperature=1.0, teacher_temperature=1.0, rest=False, soft=1.0, hard=0.0):
    """token_loss, the four sums, the gradient, and bounds on the kernel's rounding of each (the gradient's before the last one)."""
    rows, vocab = logits.shape
    device = logits.device
    w = torch.ones(rows, dtype=torch.float64, device=device) if weights is None else weights.double()
    taking = w != 0
    if labels is not None:
        taking = taking & (labels >= 0) & (labels < vocab)
    out = {"kl": [], "ce": [], "grad": [], "kl_bound": [], "ce_bound": [], "grad_bound": [], "active": []}
    for t in range(rows):
        x = logits[t].double()
        zero = torch.zeros_like(x)
        active = bool(taking[t]) and not bool((x == -math.inf).all())
        out["active"].append(active)
        if not active:
            for name, v in (("kl", 0.0), ("ce", 0.0), ("grad", zero), ("kl_bound", 0.0), ("ce_bound", 0.0), ("grad_bound", zero)):
                out[name].append(v)
            continue
        every = log_softmax(x, temperature)
        p = every.exp()
        listed = [(int(i), float(v) / teacher_temperature) for i, v in zip(ids[t], values[t]) if 0 <= int(i) < vocab]
        shift = 0.0
        if not rest:
            top = max((v for _, v in listed), default=-math.inf)
            shift = top + math.log(math.fsum(math.exp(v - top) for _, v in listed)) if math.isfinite(top) else top
        q = {}
        kl = size = 0.0
        for i, v in listed:
            log_q = -math.inf if v == -math.inf else v - shift
            each = math.exp(log_q) if log_q == log_q else math.nan
            q[i] = q.get(i, 0.0) + each
            if each != 0.0:
                kl += each * (log_q - float(every[i]))
                size += each * (abs(log_q) + abs(float(every[i])))
        mass = math.fsum(q.values())
        inside = torch.zeros_like(x, dtype=torch.bool)
        if q:
            inside[torch.tensor(list(q), device=device)] = True
        apart = torch.where(inside, torch.full_like(every, -math.inf), every)
        log_p0 = float(torch.logsumexp(apart, 0)) if bool((apart > -math.inf).any()) else -math.inf
        q0 = (1.0 - mass if not mass > 1.0 else 0.0) if rest and log_p0 > -math.inf else 0.0
        if q0 > 0:
            kl += q0 * (math.log(q0) - log_p0)
        if rest:                                       # q0 is off by what the listed probabilities are
            size += (mass + 1) * (1 + (abs(math.log(q0)) if q0 > 0 else 0.0) + (abs(log_p0) if log_p0 > -math.inf else 0.0))
        Q = mass + q0
        qs = torch.zeros_like(x)
        for i, v in q.items():
            qs[i] = v
        in_rest = zero                                 # its elements' shares of it, by differences that any size of logit keeps
        if q0 > 0:
            in_rest = log_softmax(torch.where(inside, torch.full_like(x, -math.inf), x), temperature).exp()
        grad = soft / temperature * (p * Q - qs - q0 * in_rest)
        # A step or two for every unit of an exponent, of the rest's and the whole row's reference.
        depth = (x / temperature - float((x / temperature).max())).abs().clamp(max=200.0)
        q0_off = (mass + 1) * in_rest if rest else zero
        bound = abs(soft) / temperature * ((64 + 8 * depth) * (p * Q + qs + q0 * in_rest) + 16 * q0_off)
        ce = 0.0
        if hard:
            one = log_softmax(x, 1.0)
            ce = -float(one[labels[t]])
            g = one.exp()
            deep = (x - float(x.max())).abs().clamp(max=200.0)
            bound = bound + abs(hard) * (64 + 8 * deep) * g
            g[labels[t]] -= 1
            bound[labels[t]] += abs(hard) * 8
            grad = grad + hard * g
        out["kl"].append(kl)
        out["ce"].append(ce)
        out["grad"].append(grad * w[t])
        out["kl_bound"].append(64 + 32 * size)
        out["ce_bound"].append(64 + 32 * abs(ce) if hard else 0.0)
        out["grad_bound"].append(bound * w[t].abs())
    tensor = lambda v: torch.tensor(v, dtype=torch.float64, device=device)  # noqa: E731
    kl, ce = tensor(out["kl"]), tensor(out["ce"])
    active = torch.tensor(out["active"], device=device, dtype=torch.bool)
    loss = (soft * kl if soft else torch.zeros_like(kl)) + (hard * ce if hard else torch.zeros_like(ce))
    kl_bound, ce_bound = ULP * tensor(out["kl_bound"]), ULP * tensor(out["ce_bound"])
    none = torch.zeros_like(kl)
    token_bound = (abs(soft) * kl_bound if soft else none) + (abs(hard) * ce_bound if hard else none) + 2 * ULP * loss.abs()
    w = torch.where(active, w, torch.zeros_like(w))
    sums = torch.stack([(w * loss).sum(), (w * kl).sum(), (w * ce).sum(), w.sum()])
    sums_bound = torch.stack([(w.abs() * b).sum() for b in (token_bound, kl_bound, ce_bound, none)]) + 4 * ULP * sums.abs()
    empty = torch.zeros((0, vocab), dtype=torch.float64, device=device)
    return {"token_loss": loss, "token_bound": token_bound, "sums": sums, "sums_bound": sums_bound,
            "dlogits": torch.stack(out["grad"]) if rows else empty,
            "grad_bound": ULP * torch.stack(out["grad_bound"]) + 1e-36 if rows else empty, "active": active}


def log_softmax(x, temperature):
    """The difference first: exact also where the largest logit is huge."""
    low = (x - x.max()) / temperature
    return low - torch.log(torch.exp(low).sum())


def norm(total, gain=None, eps=1e-6):
    """(y, rstd) of the stream as it is kept."""
    s = total.double()
    rstd = 1 / torch.sqrt(s.square().mean(1) + eps)
    y = s * rstd[:, None]
    return (y if gain is None else y * gain.double()), rstd


def norm_bound(cols):
    """What rstd may be off, relative: sums of squares along a thread, of at most every 32nd column, and between threads."""
    return ULP * ((cols / 32 + 24) / 2 + 6)


def norm_backward(dy, total, rstd, gain=None, d_total=None):
    """(dx, dgain, and bounds on the kernel's rounding of both before the last one)."""
    rows, cols = dy.shape
    d, r = dy.double(), rstd.double()[:, None]
    n = total.double() * r
    g = d if gain is None else d * gain.double()
    mean = (g * n).sum(1, keepdim=True) / max(cols, 1)
    dx = r * (g - n * mean)
    if d_total is not None:
        dx = dx + d_total.double()
    size = (g * n).abs().sum(1, keepdim=True) / max(cols, 1)
    dx_bound = ULP * (r * (8 * g.abs() + n.abs() * (8 * mean.abs() + (cols / 32 + 24) * size)) + 2 * dx.abs())
    return dx, (d * n).sum(0), dx_bound, ULP * (rows / 32 + 64) * (d * n).abs().sum(0)
