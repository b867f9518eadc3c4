"""The trainers' operators in 64 bits on the CPU, row by row and element by element: what the GPU's results are held to."""

import math

import torch

NAN, INF = math.nan, math.inf


def logprobs(x, targets, scale=1.0, top=0):
    """x [rows, vocab] of any type, targets int64 or None -> dict of float64 (ids int64) results."""
    x = x.double().cpu()
    rows, vocab = x.shape
    out = dict(logprob=torch.zeros(rows, dtype=torch.float64), entropy=torch.zeros(rows, dtype=torch.float64),
               norm=torch.zeros(rows, 2, dtype=torch.float64), top_ids=torch.full((rows, top), -1, dtype=torch.int64),
               top_logprobs=torch.full((rows, top), -INF, dtype=torch.float64))
    for r in range(rows):
        t = 0 if targets is None else int(targets[r])
        if t < 0:
            continue
        row = x[r]
        m = row.max()
        bad = bool(torch.isnan(row).any()) or m == INF
        rank = torch.where(torch.isnan(row), torch.full_like(row, INF), row)
        order = sorted(range(vocab), key=lambda i: (not math.isnan(row[i]), -float(rank[i]), i)) if vocab <= 64 or bad else \
            torch.argsort(-row, stable=True).tolist()
        k = min(top, vocab)
        out["top_ids"][r, :k] = torch.tensor(order[:k], dtype=torch.int64)
        if bad:
            out["logprob"][r], out["entropy"][r], out["norm"][r] = NAN, NAN, NAN
            out["top_logprobs"][r, :k] = NAN
            continue
        if m == -INF:
            out["logprob"][r], out["norm"][r] = NAN if t >= vocab else -INF, torch.tensor([-INF, 0.0], dtype=torch.float64)
            continue
        z = (row - m) * scale
        e = torch.exp(z)
        S = e.sum()
        lp = z - torch.log(S)
        p = e / S
        out["logprob"][r] = lp[t] if t < vocab else NAN
        out["entropy"][r] = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum()
        out["norm"][r] = torch.stack([m, S])
        out["top_logprobs"][r, :k] = lp[out["top_ids"][r, :k]]
    return out


def gradient(x, targets, g, h=None, scale=1.0):
    """Gradient of sum(g logprob + h entropy) by x."""
    x = x.double().cpu()
    rows, vocab = x.shape
    out = torch.zeros(rows, vocab, dtype=torch.float64)
    for r in range(rows):
        t, row = int(targets[r]), x[r]
        if t < 0:
            continue
        m = row.max()
        if t >= vocab or torch.isnan(row).any() or m == INF:
            out[r] = NAN
            continue
        if m == -INF:
            continue
        lp = torch.log_softmax((row - m) * scale, 0)
        p = torch.exp(lp)
        one = torch.zeros_like(p)
        one[t] = 1.0
        y = float(g[r]) * (one - p)
        if h is not None:
            H = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum()
            y = y - float(h[r]) * torch.where(p > 0, p * (lp + H), torch.zeros_like(p))
        out[r] = y * scale
    return out


def job_losses(offsets, targets, logprob, weights):
    losses, rows = [], torch.zeros(len(logprob), dtype=torch.float64)
    for lo, hi in zip(offsets[:-1], offsets[1:]):
        w = [0.0 if targets is not None and targets[r] < 0 else 1.0 if weights is None else float(weights[r]) for r in range(lo, hi)]
        total = math.fsum(w)
        losses.append(-math.fsum(a * float(logprob[lo + i]) for i, a in enumerate(w) if a) / total if total else NAN)
        for i, a in enumerate(w):
            rows[lo + i] = -a / total if a else 0.0
    return torch.tensor(losses, dtype=torch.float64), rows


def adamw(p, g, m, v, lr, betas, eps, weight_decay, step, grad_scale=1.0):
    """The step's new (p, m, v) in float64; `step` steps were taken before."""
    b1, b2 = betas
    g = g.double() * grad_scale
    m = b1 * m.double() + (1 - b1) * g
    v = b2 * v.double() + (1 - b2) * g * g
    t = step + 1
    p = p.double() * (1 - lr * weight_decay) - lr / (1 - b1 ** t) * m / (torch.sqrt(v) / math.sqrt(1 - b2 ** t) + eps)
    return p, m, v
