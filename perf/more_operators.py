"""More of what a trainer on the scheduler's GPU has it compute, as measurable cases.

Three operators, each on its own:

    sample      tokens drawn from rows of logits with given random numbers: temperature, top-k, top-p, min-p
    clip        the norms of jobs' gradients over many tensors, and the gradients times the factors that these give
    step        the norms and one AdamW step that applies the factors as it reads the gradients

``own`` chooses between elementary torch operations and the framework's kernels.
"""

from __future__ import annotations

import math
import random

import torch

own = False

BLOCK = 256          # tensors begin at multiples of this in the allocation that holds them
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZES = {"fp32": 4, "bf16": 2, "fp16": 2}
NONE = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)


def _rows(name, rows, vocab, dtype, **more):
    """`mixed`: every row has numbers of its own, `temperature` .. `min_p` being those of some of them, and some rows are greedy."""
    case = dict(kind="sample", rows=rows, vocab=vocab, dtype=dtype, pad=0, mixed=False, masked=False, missing=0.0, **NONE)
    case.update(more)
    if name is not None:
        case["name"] = name
    return case


def _tensors(name, kind, tensors, largest, dtype, **more):
    case = dict(kind=kind, tensors=tensors, largest=largest, smallest=1, dtype=dtype, master=False, groups=1, idle=False, max_norm=1.0)
    case.update(more)
    if name is not None:
        case["name"] = name
    return case


def listed():
    return [
        # One token of one sequence, as a served model draws it. Latency is all there is.
        _rows("sample 1 x 32768", 1, 32768, "bf16", temperature=0.7, top_k=50, top_p=0.95),
        # A batch of sequences with logits kept in fp32, an odd vocabulary with padding columns behind it.
        _rows("sample 64 x 130001 fp32", 64, 130_001, "fp32", pad=47, temperature=0.8, top_p=0.9),
        # A larger batch in which every request has its own numbers, padded vocabulary masked, a tenth of the sequences ended.
        _rows("sample 512 x 65536 mixed", 512, 65_536, "bf16", mixed=True, masked=True, missing=0.1, temperature=0.9, top_k=40, top_p=0.95, min_p=0.05),
        # A policy's rollouts, drawn from the model's whole distribution.
        _rows("sample 4096 x 128000", 4096, 128_000, "bf16"),
        # Answers of the scheduler's own kind of job, a class head: many rows of a few classes.
        _rows("sample 200000 x 10 fp32", 200_000, 10, "fp32", top_p=0.95),
        # 160 small jobs, each clipped by its own norm, one in five without cores.
        _tensors("clip 320 small fp32", "clip", 320, 20_000, "fp32", groups=160, idle=True),
        # One model's gradients in bf16.
        _tensors("clip 300 bf16", "clip", 300, 8_000_000, "bf16"),
        # The small jobs' whole step.
        _tensors("step 320 small fp32", "step", 320, 20_000, "fp32", groups=160, idle=True),
        # Mixed precision: weights and gradients in bf16, master weights and states in fp32, two models.
        _tensors("step 300 bf16 master", "step", 300, 8_000_000, "bf16", master=True, groups=2),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: the operators in turn by chance, sizes over their whole range."""
    kind = rng.choice(["sample", "sample", "sample", "clip", "step"])
    if kind != "sample":
        tensors = _log_int(rng, 1, 500)
        dtype = rng.choice(["fp32", "bf16", "fp16"])
        return _tensors(None, kind, tensors, _log_int(rng, 40, min(60_000_000, 1_200_000_000 // tensors)), dtype, smallest=rng.choice([1, 100]),
                        master=kind == "step" and dtype != "fp32" and rng.random() < 0.5, groups=rng.choice([1, 2, max(1, tensors // 2)]),
                        idle=rng.random() < 0.3, max_norm=rng.choice([0.1, 1.0, 1e9]))
    vocab = _log_int(rng, 2, 262_144)
    dtype = rng.choice(["fp32", "bf16", "bf16", "fp16"])
    rows = _log_int(rng, 1, min(200_000, 1_000_000_000 // SIZES[dtype] // vocab))
    numbers = dict(temperature=rng.choice([1.0, 0.7, 1.3]), top_k=rng.choice([0, 0, 1, 20, 50, 1000]), top_p=rng.choice([1.0, 1.0, 0.9, 0.95, 0.99]),
                   min_p=rng.choice([0.0, 0.0, 0.05]))
    if rng.random() < 0.25:
        numbers = dict(NONE, temperature=numbers["temperature"])
    return _rows(None, rows, vocab, dtype, pad=rng.choice([0, 0, 1, 8, 47]), mixed=rng.random() < 0.3, masked=vocab > 100 and rng.random() < 0.4,
                 missing=rng.choice([0.0, 0.0, 0.1, 0.5]), **numbers)


# ---- inputs ----

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _prepare_rows(case, seed):
    g, n, v = _generator(seed), case["rows"], case["vocab"]
    u = lambda *s: torch.rand(*s, generator=g, device="cuda")   # noqa: E731
    x = torch.randn(n, v + case["pad"], generator=g, device="cuda", dtype=TYPES[case["dtype"]]).mul_(2.0)[:, :v]
    # A text's rows: a handful of likely tokens, from one that is nearly certain to as good as none among a large vocabulary.
    likely = torch.randint(v, (n, 12), generator=g, device="cuda")
    height = (12.0 + 10.0 * u(n, 1)) * math.log(v) / math.log(128_000.0) - torch.empty(n, 12, device="cuda").exponential_(0.4, generator=g)
    every = torch.arange(n, device="cuda")
    for j in range(likely.shape[1]):                         # one after the other: a token may be named twice
        x[every, likely[:, j]] = height[:, j].to(x.dtype)
    if case["masked"]:
        x[:, v - v // 50:] = -math.inf                       # columns that pad the vocabulary
    uniform = u(n)
    numbers = {name: case[name] for name in NONE}
    if case["mixed"]:
        pick = lambda value, other: torch.where(u(n) < 0.7, value, other)   # noqa: E731
        numbers = {"temperature": pick(case["temperature"], 0.0) * (0.8 + 0.4 * u(n)), "top_k": pick(case["top_k"], 0).to(torch.int32),
                   "top_p": pick(case["top_p"], 1.0).float(), "min_p": pick(case["min_p"], 0.0).float()}
    uniform = torch.where(u(n) < case["missing"], -1.0, uniform)   # sequences that have ended
    return dict(case, logits=x, uniform=uniform, **numbers)


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


def _prepare_tensors(case, seed):
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
    t, group_of = TYPES[case["dtype"]], _group_of(case)
    # Some of the jobs are beyond their largest norm, and their gradients differ in size from layer to layer.
    group = torch.tensor(group_of, device="cuda")[tensor_of]
    per_group = torch.exp(1.5 * torch.randn(case["groups"], generator=g, device="cuda"))
    elements = torch.zeros(case["groups"], device="cuda").index_add_(0, group, inside.sum(1).float())
    size = torch.exp(torch.randn(nb, 1, generator=g, device="cuda")) * (per_group / elements.sqrt())[group][:, None]
    st = dict(case, inside=inside, group=group, g=(flat(1.0) * size).to(t),
              active=torch.tensor([0 if case["idle"] and k % 5 == 4 else 1 + k % 3 for k in range(case["groups"])], dtype=torch.int32, device="cuda"))
    hyper = _hyper(case)
    if case["kind"] == "clip":
        st["clipped"] = torch.zeros_like(st["g"])
    else:
        w = flat(0.05)
        st["p"], st["master"] = w.to(t), w if case["master"] else None
        st["m"], st["v"] = flat(0.3) * size, (flat(0.7) * size).square_() + 0.01 * size * size * inside
        st["hyper"] = torch.tensor([[h["lr"], *h["betas"], h["eps"], h["weight_decay"]] for h in hyper], dtype=torch.float64, device="cuda")
        st["step"] = torch.tensor([h["step"] for h in hyper], dtype=torch.float64, device="cuda")
    if own:
        import paper_1802_04819_b200 as slaq
        cut = lambda x: [x.view(-1)[BLOCK * a: BLOCK * a + n] for a, n in zip(at, numels)]   # noqa: E731
        grads = cut(st["g"])
        st["norms"] = slaq.GradNorms(grads, group_of, out=cut(st["clipped"]) if case["kind"] == "clip" else None)
        if case["kind"] == "step":
            st["plan"] = slaq.AdamW(cut(st["p"]), grads, group_of, hyper, masters=cut(st["master"]) if case["master"] else None,
                                    exp_avg=cut(st["m"]), exp_avg_sq=cut(st["v"]))
    return st


def prepare(case, seed):
    return (_prepare_rows if case["kind"] == "sample" else _prepare_tensors)(case, seed)


# ---- the operators in elementary operations ----

def _number(st, name, lo, hi, dtype):
    """A row's number: the rows' own, or one for all."""
    x = st[name]
    return x[lo:hi].to(dtype) if torch.is_tensor(x) else torch.full((hi - lo,), x, dtype=dtype, device="cuda")


def _filtered(st):
    return st["mixed"] or any(st[name] != NONE[name] for name in ("top_k", "top_p", "min_p"))


def _sample_block(st, lo, hi):
    """Which tokens are kept and which of them is drawn are decided in 64 bits: in a large vocabulary every other sum lies next to a border."""
    x, u = st["logits"][lo:hi].float(), st["uniform"][lo:hi]
    v, asked = st["vocab"], u >= 0
    t = _number(st, "temperature", lo, hi, torch.float64)
    greedy = t == 0
    m = x.amax(1, keepdim=True)
    w = ((x.double() - m.double()) / torch.where(greedy, 1.0, t)[:, None]).exp()
    total = w.sum(1)
    kept = None
    if _filtered(st):
        k, p, q = _number(st, "top_k", lo, hi, torch.int64), _number(st, "top_p", lo, hi, torch.float64), _number(st, "min_p", lo, hi, torch.float64)
        by_size, order = x.sort(dim=1, descending=True, stable=True)        # equal ones stay in the order of their ids
        sizes = w.gather(1, order)
        sums = sizes.cumsum(1)
        before = torch.cat([torch.zeros_like(sums[:, :1]), sums[:, :-1]], 1)
        k = torch.where(k > 0, k.clamp_max(v), v)
        enough = torch.where(p < 1, p * sums.gather(1, k[:, None] - 1)[:, 0], math.inf)
        rank = torch.arange(v, device="cuda")[None, :]
        keep = (rank < k[:, None]) & (before < enough[:, None]) & (sizes >= q[:, None]) & (by_size > -math.inf)
        keep &= ~greedy[:, None] | (rank == 0)
        kept = torch.where(asked, keep.sum(1), 0).to(torch.int32)
        w = w * torch.zeros_like(w).scatter_(1, order, keep.double())
    sums = w.cumsum(1)
    token = (sums <= u.double()[:, None] * sums[:, -1:]).sum(1).clamp_max(v - 1)[:, None]
    mine = torch.where(greedy, 0.0, w.gather(1, token)[:, 0].log())
    out = {"token": torch.where(asked, token[:, 0], -1),
           "logprob": torch.where(asked, mine - torch.where(greedy, 0.0, total.log()), 0.0).float(),
           "kept_logprob": torch.where(asked, mine - torch.where(greedy, 0.0, sums[:, -1].log()), 0.0).float()}
    return out if kept is None else dict(out, kept=kept)


def _sample(st):
    step = max(1, 64_000_000 // st["vocab"])
    parts = [_sample_block(st, lo, min(st["rows"], lo + step)) for lo in range(0, st["rows"], step)]
    return {name: torch.cat([p[name] for p in parts]) for name in parts[0]}


def _norms(st):
    n, on = st["groups"], st["active"] > 0
    squares = st["g"].float().square().sum(1).double()       # of a block's 256 elements
    norm = torch.zeros(n, dtype=torch.float64, device="cuda").index_add_(0, st["group"], squares).sqrt()
    factor = torch.where(norm > st["max_norm"], st["max_norm"] / norm, 1.0)
    return torch.where(on, norm, 0.0).float(), torch.where(on, factor, 1.0).float(), on


def _clip(st):
    norm, factor, on = _norms(st)
    clipped = st["g"].float() * factor[st["group"]][:, None]
    st["clipped"].copy_(torch.where(on[st["group"]][:, None], clipped.to(st["g"].dtype), st["clipped"]))
    return {"norm": norm, "factor": factor, "clipped": st["clipped"]}


def _step(st):
    norm, factor, active = _norms(st)
    lr, b1, b2, eps, decay = st["hyper"].unbind(1)
    t = st["step"] + 1
    coefs = [b1, 1 - b1, b2, 1 - b2, 1 / (1 - b2 ** t).sqrt(), eps, 1 - lr * decay, lr / (1 - b1 ** t), factor]
    b1, a1, b2, a2, correct, eps, keep, size, factors = (c.float()[st["group"]][:, None] for c in coefs)
    on = active[st["group"]][:, None]
    g = st["g"].float() * factors
    p = st["p"].float() if st["master"] is None else st["master"]
    m = b1 * st["m"] + a1 * g
    v = b2 * st["v"] + a2 * (g * g)
    p = p * keep - size * (m / (v.sqrt() * correct + eps))
    put = lambda name, x: st[name].copy_(torch.where(on, x, st[name]))   # noqa: E731
    put("p", p.to(st["p"].dtype))
    if st["master"] is not None:
        put("master", p)
    put("m", m)
    put("v", v)
    st["step"].add_(active)
    return {"norm": norm, "factor": factor}


# ---- the framework's calls ----

def _own(st):
    import paper_1802_04819_b200 as slaq
    if st["kind"] == "sample":
        given = {name: st[name] for name in ("top_k", "top_p", "min_p")} if _filtered(st) else {}
        r = slaq.sample_tokens(st["logits"], st["uniform"], temperature=st["temperature"], **given)
        out = {"token": r.token, "logprob": r.logprob, "kept_logprob": r.kept_logprob}
        return dict(out, kept=r.kept) if given else out
    norm, factor = st["norms"].measure(st["max_norm"], active=st["active"])
    if st["kind"] == "clip":
        st["norms"].apply(factor, active=st["active"])
        return {"norm": norm, "factor": factor, "clipped": st["clipped"]}
    st["plan"].step(st["active"], factors=factor)
    return {"norm": norm, "factor": factor}


def run(st):
    out = _own(st) if own else {"sample": _sample, "clip": _clip, "step": _step}[st["kind"]](st)
    if st["kind"] == "step":
        out = dict(out, p=st["p"], m=st["m"], v=st["v"])
        if st["master"] is not None:
            out["master"] = st["master"]
    return out


def work(case):
    e = SIZES[case["dtype"]]
    if case["kind"] == "sample":
        asked = (1.0 - case["missing"]) * case["rows"]
        return {"bytes": asked * case["vocab"] * e + case["rows"] * (20.0 + 4.0 * case["mixed"] * 4), "flops": 4.0 * asked * case["vocab"]}
    on = [not (case["idle"] and k % 5 == 4) for k in range(case["groups"])]
    n = sum(n for n, k in zip(_numels(case), _group_of(case)) if on[k])
    if case["kind"] == "clip":
        return {"bytes": 2.0 * e * n, "flops": 3.0 * n}
    return {"bytes": (3.0 * e + 16.0 + (8.0 - e) * case["master"]) * n, "flops": 17.0 * n}


# ---- the definitions in 64 bits ----

def _exact_sample_block(st, lo, hi):
    x, u, n, v = st["logits"][lo:hi].double(), st["uniform"][lo:hi].double(), hi - lo, st["vocab"]
    t = _number(st, "temperature", lo, hi, torch.float64)
    greedy, off = t == 0.0, u < 0.0
    z = x / torch.where(greedy, 1.0, t)[:, None]
    share = torch.softmax(z, 1)                                # of all tokens
    kept = None
    if _filtered(st):
        falling, ids = torch.sort(x, dim=1, descending=True, stable=True)
        first = torch.gather(share, 1, ids)
        mass = torch.cumsum(first, 1)
        length = (falling != -math.inf).sum(1)
        k = _number(st, "top_k", lo, hi, torch.int64)
        length = torch.where(k > 0, torch.minimum(length, k), length)
        p = _number(st, "top_p", lo, hi, torch.float64)
        of_k = mass.gather(1, length[:, None] - 1)
        enough = 1 + torch.searchsorted(mass, p[:, None] * of_k)[:, 0]      # mass[j - 1] < p S <= mass[j]
        length = torch.where(p < 1.0, torch.minimum(length, enough), length)
        q = _number(st, "min_p", lo, hi, torch.float64)
        length = torch.minimum(length, (first >= q[:, None] * first[:, :1]).sum(1))
        length = torch.where(greedy, 1, length)
        kept = length.masked_fill(off, 0).to(torch.int32)
        rank = torch.empty_like(ids).scatter_(1, ids, torch.arange(v, device="cuda").expand(n, v))
        inside = share.masked_fill(rank >= length[:, None], 0.0)
    else:
        inside = share
    running = torch.cumsum(inside, 1)
    every = running[:, -1]
    token = torch.searchsorted(running, (u * every)[:, None], right=True)[:, 0].clamp_max(v - 1)
    lse = torch.logsumexp(z, 1)
    own_z = z.gather(1, token[:, None])[:, 0]
    none = lambda y: y.masked_fill(off | greedy, 0.0)   # noqa: E731
    kept_lse = torch.logsumexp(z.masked_fill(inside == 0.0, -math.inf), 1) if kept is not None else lse
    out = {"token": token.masked_fill(off, -1), "logprob": none(own_z - lse), "kept_logprob": none(own_z - kept_lse)}
    return out if kept is None else dict(out, kept=kept)


def _exact_sample(st):
    step = max(1, 40_000_000 // st["vocab"])
    parts = [_exact_sample_block(st, lo, min(st["rows"], lo + step)) for lo in range(0, st["rows"], step)]
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}


def _exact_norms(st):
    nb, norm = st["g"].shape[0], torch.zeros(st["groups"], dtype=torch.float64, device="cuda")
    for lo in range(0, nb, 1 << 18):
        s = slice(lo, min(nb, lo + (1 << 18)))
        norm.index_add_(0, st["group"][s], (st["g"][s].double() ** 2).sum(1))
    norm = torch.sqrt(norm)
    on = st["active"] > 0
    factor = torch.clamp(st["max_norm"] / norm, max=1.0)
    return norm.masked_fill(~on, 0.0), factor.masked_fill(~on, 1.0), on


def _exact_tensors(st):
    norm, factor, on = _exact_norms(st)
    clip = st["kind"] == "clip"
    names = ["clipped"] if clip else ["p", "m", "v"] + ["master"] * (st["master"] is not None)
    parts = {n: [] for n in names}
    if not clip:
        lr, b1, b2, eps, decay = st["hyper"].unbind(1)
        t = st["step"] + 1
    for lo in range(0, st["g"].shape[0], 1 << 16):
        s = slice(lo, lo + (1 << 16))
        k = st["group"][s]
        c = lambda x: x[k][:, None]   # noqa: E731
        old = {n: st[n][s].double() for n in names}
        g = st["g"][s].double() * c(factor)
        if clip:
            new = {"clipped": g}
        else:
            m = c(b1) * old["m"] + (1 - c(b1)) * g
            v = c(b2) * old["v"] + (1 - c(b2)) * g ** 2
            w = old["master"] if "master" in old else old["p"]
            w = w - c(lr) * c(decay) * w - c(lr) * (m / (1 - c(b1 ** t))) / (torch.sqrt(v / (1 - c(b2 ** t))) + c(eps))
            new = {"p": w, "master": w, "m": m, "v": v}
        for n in names:
            parts[n].append(torch.where(c(on), new[n], old[n]))
    out = {"norm": norm, "factor": factor}
    for n in names:
        out[n] = torch.cat(parts.pop(n))
    return out


def exact(case, seed):
    st = prepare(case, seed)
    return _exact_sample(st) if case["kind"] == "sample" else _exact_tensors(st)
