"""What a trainer on the scheduler's GPU has it compute, as measurable cases.

Five operators, each on its own:

    logprobs    log probabilities of given tokens, with the entropy and the top alternatives of their rows
    grad        the gradient of those log probabilities and entropies with respect to the logits
    loss        log probabilities and gradient in one call, where the rows' factors are known beforehand
    jobs        the factors of the rows in their jobs' mean losses, and those losses, as the scheduler takes them
    adamw       one AdamW step over the tensors of many jobs, states in 32 or in 8 bits

``own`` chooses between elementary torch operations and the framework's kernels.
"""

from __future__ import annotations

import math
import random

import torch

own = False

BLOCK = 256          # elements of a tensor that share the scale of an 8-bit state
E4M3_MAX = 448.0
TINY = 2.0 ** -100   # a block whose largest value is below this has nothing worth keeping
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZES = {"fp32": 4, "bf16": 2, "fp16": 2}


def _rows(name, kind, rows, vocab, dtype, **more):
    case = dict(kind=kind, rows=rows, vocab=vocab, dtype=dtype, pad=0, top=0, scale=1.0, masked=False, missing=0.0,
                entropy=True)
    case.update(more)
    if name is not None:
        case["name"] = name
    return case


def _jobs(name, jobs, longest, weighted):
    case = dict(kind="jobs", jobs=jobs, longest=longest, weighted=weighted)
    if name is not None:
        case["name"] = name
    return case


def _adamw(name, tensors, largest, dtype, bits, **more):
    case = dict(kind="adamw", tensors=tensors, largest=largest, smallest=1, dtype=dtype, bits=bits, master=False,
                groups=2, idle=False)
    case.update(more)
    if name is not None:
        case["name"] = name
    return case


def listed():
    return [
        # One generated token: its log probability and five alternatives. Latency is all there is.
        _rows("logprobs 1 x 32768", "logprobs", 1, 32768, "bf16", top=5),
        # A batch of generated tokens at a sampling temperature, logits kept in fp32, an odd vocabulary with padding
        # columns behind it.
        _rows("logprobs 64 x 130001 fp32", "logprobs", 64, 130001, "fp32", pad=47, top=20, scale=1.0 / 0.7),
        # Scoring of long texts: what a job reports when it evaluates, a tenth of the rows prompts or padding.
        _rows("logprobs 8192 x 65536", "logprobs", 8192, 65536, "bf16", missing=0.1),
        # The backward pass of a policy's update with an entropy bonus; odd rows lie at every alignment.
        _rows("grad 2048 x 50001", "grad", 2048, 50001, "bf16"),
        # Class heads of the scheduler's own kind of job (multinomial logistic regression): many rows of a few classes.
        _rows("grad 200000 x 10 fp32", "grad", 200_000, 10, "fp32", entropy=False),
        # A training step's loss and gradient over a batch of sequences, padded vocabulary masked, prompts left out.
        _rows("loss 4096 x 128000", "loss", 4096, 128_000, "bf16", masked=True, missing=0.1),
        # A small job's training step.
        _rows("loss 200 x 5000 fp16", "loss", 200, 5000, "fp16"),
        # The cluster experiment's 160 jobs, a batch of a few thousand tokens each.
        _jobs("jobs 160", 160, 4096, True),
        # The scalability experiment's 4,000 jobs.
        _jobs("jobs 4000", 4000, 2000, False),
        # 160 small jobs' weights in one step, every job at a step of its own, one in five without cores.
        _adamw("adamw 320 small fp32", 320, 20_000, "fp32", 32, groups=160, idle=True),
        # Mixed precision: weights and gradients in bf16, master weights and states in fp32.
        _adamw("adamw 300 bf16 master", 300, 8_000_000, "bf16", 32, master=True),
        # States in 8 bits, the largest model that fits beside a scheduler.
        _adamw("adamw 400 bf16 8-bit", 400, 8_000_000, "bf16", 8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: the operators in turn by chance, sizes over their whole range."""
    kind = rng.choice(["logprobs", "logprobs", "grad", "loss", "loss", "jobs", "adamw", "adamw", "adamw"])
    if kind == "jobs":
        jobs = _log_int(rng, 1, 20_000)
        return _jobs(None, jobs, _log_int(rng, 1, min(4_000_000, 16_000_000 // jobs)), rng.random() < 0.5)
    if kind == "adamw":
        tensors = _log_int(rng, 1, 500)
        bits = rng.choice([8, 32])
        dtype = rng.choice(["fp32", "bf16", "fp16"])
        return _adamw(None, tensors, _log_int(rng, 40, min(100_000_000, 2_000_000_000 // tensors)), dtype, bits,
                      smallest=rng.choice([1, 100]), master=dtype != "fp32" and rng.random() < 0.5,
                      groups=rng.choice([1, 2, max(1, tensors // 2)]), idle=rng.random() < 0.3)
    vocab = _log_int(rng, 2, 262_144)
    dtype = rng.choice(["fp32", "bf16", "bf16", "fp16"])
    rows = _log_int(rng, 1, min(200_000, 1_000_000_000 // SIZES[dtype] // vocab))
    return _rows(None, kind, rows, vocab, dtype, pad=rng.choice([0, 0, 1, 8, 47]),
                 top=rng.choice([0, 1, 5, 20, 32]) if kind == "logprobs" else 0, scale=rng.choice([1.0, 1.0, 1.0 / 0.7]),
                 masked=vocab > 100 and rng.random() < 0.4, missing=rng.choice([0.0, 0.0, 0.1, 0.5]),
                 entropy=kind == "logprobs" or (kind == "grad" and rng.random() < 0.5))


# ---- inputs ----

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _prepare_rows(case, seed):
    g, n, v = _generator(seed), case["rows"], case["vocab"]
    u = lambda *s: torch.rand(*s, generator=g, device="cuda")   # noqa: E731
    x = torch.randn(n, v + case["pad"], generator=g, device="cuda", dtype=TYPES[case["dtype"]]).mul_(2.5)[:, :v]
    likely = torch.randint(v, (n,), generator=g, device="cuda")
    every = torch.arange(n, device="cuda")
    x[every, likely] += (6.0 + 8.0 * u(n)).to(x.dtype)      # a text's rows are peaked, more or less
    if case["masked"]:
        x[:, v - v // 50:] = -math.inf                       # columns that pad the vocabulary
    other = torch.randint(v, (n,), generator=g, device="cuda")
    targets = torch.where(u(n) < 0.6, likely, other)
    targets = torch.where(u(n) < case["missing"], torch.full_like(targets, -1), targets)
    st = dict(case, logits=x, targets=targets)
    if case["kind"] == "loss":
        st["row_grad"] = torch.where(targets >= 0, -1.0 / n, 0.0)
        st["grad"] = torch.empty(n, v, dtype=x.dtype, device="cuda")
    if case["kind"] == "grad":
        m = x.float().amax(1)
        d = (x.float() - m[:, None]) * case["scale"]
        s = d.exp().sum(1)
        st["norm"] = torch.stack([m, s], 1)
        st["h"] = s.log() - (d.exp() * d.clamp_min(-1e30)).sum(1) / s
        st["g_logprob"] = torch.randn(n, generator=g, device="cuda") / n
        st["g_entropy"] = torch.full((n,), 0.01 / n, device="cuda") if case["entropy"] else None
        st["grad"] = torch.empty(n, v, dtype=x.dtype, device="cuda")
    return st


def _lengths(case):
    """Rows per job: ragged over the whole range, an empty job now and then where there are many."""
    r = random.Random(case["jobs"] * 1_000_003 + case["longest"])
    n = [_log_int(r, 1, case["longest"]) if r.random() < 0.7 else r.randint(1, case["longest"]) for _ in range(case["jobs"])]
    n[r.randrange(len(n))] = case["longest"]
    return n


def _prepare_jobs(case, seed):
    g, lengths = _generator(seed), _lengths(case)
    offsets = torch.zeros(len(lengths) + 1, dtype=torch.int64)
    offsets[1:] = torch.tensor(lengths).cumsum(0)
    rows = int(offsets[-1])
    u = lambda: torch.rand(rows, generator=g, device="cuda")   # noqa: E731
    first = torch.zeros(rows, dtype=torch.bool, device="cuda")
    first[offsets[:-1].cuda()] = True                          # every job has one row at least that counts
    targets = torch.where((u() < 0.1) & ~first, -1, 17)
    return dict(case, offsets=offsets.cuda(), targets=targets, logprob=-3.0 * u() - 1e-3,
                weights=0.5 + u() if case["weighted"] else None)


def _numels(case):
    r = random.Random(case["tensors"] * 1_000_003 + case["largest"])
    lo = min(case["smallest"], case["largest"])
    n = [_log_int(r, max(lo, case["largest"] // 2000), case["largest"]) if r.random() < 0.7 else _log_int(r, lo, max(lo, case["largest"] // 500))
         for _ in range(case["tensors"])]
    n[0] = case["largest"]
    return n


def _group_of(case):
    return [t * case["groups"] // case["tensors"] for t in range(case["tensors"])]


def _hyper(case):
    """Per group: learning rate, decays, epsilon, weight decay, steps taken so far."""
    return [dict(lr=1e-3 * (1 + k % 7), betas=(0.9, 0.999 if k % 3 else 0.95), eps=1e-8, weight_decay=0.01 * (k % 2), step=3 + 13 * k % 400)
            for k in range(case["groups"])]


def _prepare_adamw(case, seed):
    # The tensors lie in one allocation each for weights, gradients and states, every tensor at the start of a block.
    g, numels = _generator(seed), _numels(case)
    blocks = [-(-n // BLOCK) for n in numels]
    nb, at = sum(blocks), [0]
    for b in blocks:
        at.append(at[-1] + b)
    starts, counts = torch.tensor(at[:-1], device="cuda"), torch.tensor(numels, device="cuda")
    tensor_of = torch.repeat_interleave(torch.arange(len(numels), device="cuda"), torch.tensor(blocks, device="cuda"), output_size=nb)
    left = counts[tensor_of] - (torch.arange(nb, device="cuda") - starts[tensor_of]) * BLOCK
    inside = torch.arange(BLOCK, device="cuda")[None, :] < left[:, None]
    flat = lambda std: torch.randn(nb, BLOCK, generator=g, device="cuda").mul_(std).mul_(inside)   # noqa: E731
    t = TYPES[case["dtype"]]
    w = flat(0.05)
    st = dict(case, inside=inside, p=w.to(t), master=w if case["master"] else None)
    size = torch.exp(2.0 * torch.randn(nb, 1, generator=g, device="cuda")) * 1e-3      # gradients differ in size from layer to layer
    st["g"] = (flat(1.0) * size).to(t)
    m, v = flat(0.3) * size, (flat(0.7) * size).square_() + 0.01 * size * size * inside
    if case["bits"] == 32:
        st["m"], st["v"] = m, v
    else:
        (st["m"], st["m_scale"]), (st["v"], st["v_scale"]) = _to_8(m), _to_8(v.sqrt(), True)
    group_of = _group_of(case)
    st["group"] = torch.tensor(group_of, device="cuda")[tensor_of]
    hyper = _hyper(case)
    st["hyper"] = torch.tensor([[h["lr"], *h["betas"], h["eps"], h["weight_decay"]] for h in hyper], dtype=torch.float64, device="cuda")
    st["step"] = torch.tensor([h["step"] for h in hyper], dtype=torch.float64, device="cuda")
    st["active"] = torch.tensor([0 if case["idle"] and k % 5 == 4 else 1 + k % 3 for k in range(case["groups"])], dtype=torch.int32, device="cuda")
    if own:
        import paper_1802_04819_b200 as slaq
        cut = lambda x: [x.view(-1)[BLOCK * a: BLOCK * a + n] for a, n in zip(at, numels)]   # noqa: E731
        more = {}
        if case["bits"] == 8:
            scales = lambda x: [x.view(-1)[a: a + b] for a, b in zip(at, blocks)]   # noqa: E731
            more = dict(exp_avg_scale=scales(st["m_scale"]), exp_avg_sq_scale=scales(st["v_scale"]))
        st["plan"] = slaq.AdamW(cut(st["p"]), cut(st["g"]), group_of, hyper, state_bits=case["bits"],
                                masters=cut(st["master"]) if case["master"] else None, exp_avg=cut(st["m"]), exp_avg_sq=cut(st["v"]), **more)
    return st


def prepare(case, seed):
    return {"jobs": _prepare_jobs, "adamw": _prepare_adamw}.get(case["kind"], _prepare_rows)(case, seed)


# ---- the operators in elementary operations ----

def _softmax_parts(st):
    x = st["logits"].float()
    m = x.amax(1, keepdim=True)
    d = (x - m) * st["scale"]
    return x, m, d, d.exp()


def _logprobs(st):
    x, m, d, e = _softmax_parts(st)
    asked, s = st["targets"] >= 0, e.sum(1)
    none = torch.zeros_like(s)
    log_s = s.log()
    out = {"logprob": torch.where(asked, d.gather(1, st["targets"].clamp_min(0)[:, None])[:, 0] - log_s, none),
           "entropy": torch.where(asked, log_s - (e * torch.where(e > 0, d, torch.zeros_like(d))).sum(1) / s, none),
           "norm": torch.where(asked[:, None], torch.stack([m[:, 0], s], 1), torch.zeros_like(m))}
    if k := min(st["top"], st["vocab"]):
        bits = (x + 0.0).view(torch.int32).to(torch.int64)              # ordered as the values are ..
        key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) * 2 ** 20 - torch.arange(st["vocab"], device=x.device)   # .. and the lower index first
        at = key.topk(k, 1).indices
        out["top_ids"] = torch.full((x.shape[0], st["top"]), -1, dtype=torch.int32, device=x.device)
        out["top_logprobs"] = torch.full((x.shape[0], st["top"]), -math.inf, device=x.device)
        out["top_ids"][:, :k] = torch.where(asked[:, None], at.to(torch.int32), -1)
        out["top_logprobs"][:, :k] = torch.where(asked[:, None], d.gather(1, at) - log_s[:, None], -math.inf)
    return out


def _gradient(st, d, p, g, h_row, entropy, log_s):
    asked = st["targets"] >= 0
    out = p * -g[:, None]
    out.scatter_add_(1, st["targets"].clamp_min(0)[:, None], g[:, None])
    if h_row is not None:
        out -= h_row[:, None] * p * torch.where(p > 0, d - log_s[:, None] + entropy[:, None], torch.zeros_like(d))
    return torch.where(asked[:, None], out * st["scale"], torch.zeros_like(out))


def _grad(st):
    m, s = st["norm"][:, :1], st["norm"][:, 1:]
    d = (st["logits"].float() - m) * st["scale"]
    st["grad"].copy_(_gradient(st, d, d.exp() / s, st["g_logprob"], st["g_entropy"], st["h"], s[:, 0].log()))
    return st["grad"]


def _loss(st):
    _, _, d, e = _softmax_parts(st)
    s = e.sum(1, keepdim=True)
    logprob = (d.gather(1, st["targets"].clamp_min(0)[:, None]) - s.log())[:, 0]
    st["grad"].copy_(_gradient(st, d, e / s, st["row_grad"], None, None, None))
    return {"logprob": torch.where(st["targets"] >= 0, logprob, torch.zeros_like(logprob)), "grad": st["grad"]}


def _job_losses(st):
    rows, n = st["targets"].numel(), st["jobs"]
    owner = torch.repeat_interleave(torch.arange(n, device="cuda"), st["offsets"].diff(), output_size=rows)
    w = (st["targets"] >= 0).double() if st["weights"] is None else torch.where(st["targets"] >= 0, st["weights"], 0.0).double()
    total = torch.zeros(n, dtype=torch.float64, device="cuda").index_add_(0, owner, w)
    lost = torch.zeros(n, dtype=torch.float64, device="cuda").index_add_(0, owner, torch.where(w != 0, w * st["logprob"], 0.0))
    return {"row_grad": (-w / total[owner]).float(), "loss": -lost / total}


def _to_8(x, positive=False):
    """Values of a block as e4m3 times a scale; what is positive stays so."""
    most = torch.where(x.isfinite(), x.abs(), 0.0).amax(1, keepdim=True)
    kept = most >= TINY
    inverse = torch.where(kept, E4M3_MAX / most, 0.0)
    y = x * inverse
    if positive:
        y = torch.where(kept & (x > 0), y.clamp_min(2.0 ** -9), y)
    return y.to(torch.float8_e4m3fn), torch.where(kept, most / E4M3_MAX, 0.0)


def _adamw_step(st):
    eight = st["bits"] == 8
    lr, b1, b2, eps, decay = st["hyper"].unbind(1)
    active = st["active"] > 0
    t = st["step"] + 1
    coefs = [b1, 1 - b1, b2, 1 - b2, 1 / (1 - b2 ** t).sqrt(), eps, 1 - lr * decay, lr / (1 - b1 ** t)]
    b1, a1, b2, a2, correct, eps, keep, size = (c.float()[st["group"]][:, None] for c in coefs)
    on = active[st["group"]][:, None]
    g = st["g"].float()
    p = st["p"].float() if st["master"] is None else st["master"]
    m = st["m"].float() * st["m_scale"] if eight else st["m"]
    v = (st["v"].float() * st["v_scale"]).square() if eight else st["v"]
    m = b1 * m + a1 * g
    v = b2 * v + a2 * (g * g)
    r = v.sqrt()
    p = p * keep - size * (m / (r * correct + eps))
    put = lambda name, x: st[name].copy_(torch.where(on, x, st[name]))   # noqa: E731
    put("p", p.to(st["p"].dtype))
    if st["master"] is not None:
        put("master", p)
    if eight:
        for name, (x, scale) in (("m", _to_8(m)), ("v", _to_8(r, True))):
            st[name].view(torch.uint8).copy_(torch.where(on, x.view(torch.uint8), st[name].view(torch.uint8)))
            put(name + "_scale", scale)
    else:
        put("m", m)
        put("v", v)
    st["step"].add_(active)


# ---- the framework's calls ----

def _own(st):
    import paper_1802_04819_b200 as slaq
    kind = st["kind"]
    if kind == "logprobs":
        r = slaq.token_logprobs(st["logits"], st["targets"], top=st["top"], scale=st["scale"])
        out = {"logprob": r.logprob, "entropy": r.entropy, "norm": r.norm}
        return dict(out, top_ids=r.top_ids, top_logprobs=r.top_logprobs) if st["top"] else out
    if kind == "grad":
        return slaq.token_logprobs_grad(st["logits"], st["targets"], st["norm"], st["g_logprob"], entropy=st["h"],
                                        grad_entropy=st["g_entropy"], scale=st["scale"], out=st["grad"])
    if kind == "loss":
        logprob, grad = slaq.token_loss(st["logits"], st["targets"], st["row_grad"], scale=st["scale"], out=st["grad"])
        return {"logprob": logprob, "grad": grad}
    if kind == "jobs":
        return {"row_grad": slaq.job_row_grad(st["offsets"], st["targets"], st["weights"]),
                "loss": slaq.job_losses(st["offsets"], st["targets"], st["logprob"], st["weights"])}
    st["plan"].step(st["active"])


def run(st):
    kind = st["kind"]
    if own:
        out = _own(st)
    else:
        out = {"logprobs": _logprobs, "grad": _grad, "loss": _loss, "jobs": _job_losses, "adamw": _adamw_step}[kind](st)
    if kind != "adamw":
        return out
    names = ["p", "m", "v"] + ["master"] * (st["master"] is not None) + ["m_scale", "v_scale"] * (st["bits"] == 8)
    return {name: st[name] for name in names}


def work(case):
    if case["kind"] == "jobs":
        rows = sum(_lengths(case))
        return {"bytes": (8.0 + 4.0 + 4.0 + 4.0 * case["weighted"]) * rows + 16.0 * case["jobs"], "flops": 4.0 * rows}
    if case["kind"] == "adamw":
        e = SIZES[case["dtype"]]
        each = 3 * e + 8 * case["master"] - e * case["master"] + (16 if case["bits"] == 32 else 4 + 16.0 / BLOCK)
        on = [not (case["idle"] and k % 5 == 4) for k in range(case["groups"])]
        n = sum(n for n, k in zip(_numels(case), _group_of(case)) if on[k])
        return {"bytes": each * n, "flops": 14.0 * n}
    n, v, e = case["rows"], case["vocab"], SIZES[case["dtype"]]
    asked = (1.0 - case["missing"]) * n
    if case["kind"] == "logprobs":
        return {"bytes": asked * v * e + n * (8.0 + 16.0 + 8.0 * case["top"]), "flops": 7.0 * asked * v}
    return {"bytes": asked * v * e + n * v * e + n * 28.0, "flops": (8.0 if case["kind"] == "loss" else 5.0) * asked * v}


# ---- the definitions in 64 bits ----

def _exact_row_block(st, lo, hi):
    x, t = st["logits"][lo:hi].double() * float(st["scale"]), st["targets"][lo:hi]
    lse = torch.logsumexp(x, 1)
    lp = x - lse[:, None]
    p = torch.exp(lp)
    plogp = torch.where(p > 0, p * lp, 0.0)
    entropy = -plogp.sum(1)
    given = lp[torch.arange(hi - lo, device="cuda"), t.clamp_min(0)]
    off = t < 0
    if st["kind"] == "logprobs":
        m = st["logits"][lo:hi].double().max(1).values
        out = {"logprob": given.masked_fill(off, 0.0), "entropy": entropy.masked_fill(off, 0.0),
               "norm": torch.stack([m, torch.exp(lse - m * float(st["scale"]))], 1).masked_fill(off[:, None], 0.0)}
        if st["top"]:
            k = min(st["top"], st["vocab"])
            best = torch.full((hi - lo, st["top"]), -math.inf, dtype=torch.float64, device="cuda")
            best[:, :k] = lp.topk(k, 1).values
            out["top_ids"], out["top_logprobs"] = None, best.masked_fill(off[:, None], -math.inf)
        return out
    g = (st["row_grad"] if st["kind"] == "loss" else st["g_logprob"])[lo:hi].double()
    one = torch.zeros_like(p)
    one[torch.arange(hi - lo, device="cuda"), t.clamp_min(0)] = 1.0
    grad = g[:, None] * (one - p)
    if st.get("g_entropy") is not None:
        grad -= st["g_entropy"][lo:hi].double()[:, None] * (plogp + p * entropy[:, None])
    grad = (grad * float(st["scale"])).masked_fill(off[:, None], 0.0)
    return {"logprob": given.masked_fill(off, 0.0), "grad": grad} if st["kind"] == "loss" else {"grad": grad}


def _exact_rows(st):
    step, parts = max(1, 60_000_000 // st["vocab"]), []
    for lo in range(0, st["rows"], step):
        block = _exact_row_block(st, lo, min(st["rows"], lo + step))
        parts.append({k: None if v is None else v.to("cpu" if v.numel() > 10 ** 8 else "cuda") for k, v in block.items()})
    out = {k: None if parts[0][k] is None else torch.cat([p[k] for p in parts]) for k in parts[0]}
    return out["grad"] if st["kind"] == "grad" else out


def _exact_jobs(st):
    off, t, lp = st["offsets"].tolist(), st["targets"], st["logprob"].double()
    w = ((t >= 0) * (1.0 if st["weights"] is None else st["weights"].double())).double()
    loss, row = [], torch.empty_like(w)
    for lo, hi in zip(off[:-1], off[1:]):
        total = w[lo:hi].sum()
        loss.append(-(w[lo:hi] * lp[lo:hi]).sum() / total)
        row[lo:hi] = -w[lo:hi] / total
    return {"row_grad": row, "loss": torch.stack(loss)}


def _exact_adamw(st):
    nb, out = st["p"].shape[0], {}
    names = ["p", "m", "v"] + ["master"] * (st["master"] is not None) + ["m_scale", "v_scale"] * (st["bits"] == 8)
    parts = {n: [] for n in names}
    lr, b1, b2, eps, decay = st["hyper"].unbind(1)
    t = st["step"] + 1
    for lo in range(0, nb, 1 << 16):
        s = slice(lo, min(nb, lo + (1 << 16)))
        k = st["group"][s]
        c = lambda x: x[k][:, None]   # noqa: E731
        old = {n: st[n][s].double() for n in names}
        m, v, g = old["m"], old["v"], st["g"][s].double()
        if st["bits"] == 8:
            m, v = m * old["m_scale"], (v * old["v_scale"]) ** 2
        m = c(b1) * m + (1 - c(b1)) * g
        v = c(b2) * v + (1 - c(b2)) * g ** 2
        w = old["master"] if "master" in old else old["p"]
        w = w - c(lr) * c(decay) * w - c(lr) * (m / (1 - c(b1 ** t))) / (torch.sqrt(v / (1 - c(b2 ** t))) + c(eps))
        new = {"p": w, "master": w, "m": m, "v": v, "m_scale": m.abs().amax(1, keepdim=True) / E4M3_MAX,
               "v_scale": v.sqrt().amax(1, keepdim=True) / E4M3_MAX}
        for n in names:
            parts[n].append(torch.where(c(st["active"] > 0), new[n], old[n]).to(torch.float64))
    for n in names:   # an 8-bit code stands for a rounded value: it has no exact one
        out[n] = None if st["bits"] == 8 and n in ("m", "v") else torch.cat(parts[n])
        parts[n] = None
    return out


def exact(case, seed):
    st = prepare(case, seed)
    return {"jobs": _exact_jobs, "adamw": _exact_adamw}.get(case["kind"], _exact_rows)(st)
