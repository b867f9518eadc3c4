"""The AdamW step over many tensors against 64 bits.

Tolerances (u = 2^-24): m is the sum of two products, each rounded, with rounded factors: 3u (|b1 m| + |a1 g|); v the same with
two more; the new weight's decay 3u|p|, its step 12u of the step (root, correction, sum, division, product, m's and v's own), one
rounding to the type.  States in 8 bits: half a step of e4m3 (2^-4 of the value), or 2^-10 of the scale below its normal range,
and the smallest code where a second moment would vanish."""

import math

import numpy as np
import pytest
import torch

import token_rows as ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
KINDS = [(torch.float32, torch.float32, False), (torch.bfloat16, torch.bfloat16, False), (torch.bfloat16, torch.bfloat16, True),
         (torch.bfloat16, torch.float32, True), (torch.float16, torch.float16, False), (torch.float16, torch.float32, False)]
SIZES = [1, 7, 8, 255, 256, 257, 1023, 1024, 1025, 0, 5000, 40_003, 3]


@pytest.fixture(scope="module")
def slaq():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_1802_04819_b200 as mod
    mod.build()
    return mod


def _cut(sizes, dtype, gen, std, shift=0):
    """Tensors of these sizes, one behind the other from element `shift` of one buffer: all alignments."""
    flat = (torch.randn(sum(sizes) + shift, generator=gen) * std).to(dtype).cuda()
    at = np.cumsum([shift] + list(sizes))
    return [flat[a: a + n] for a, n in zip(at, sizes)]


def _near(got, want, tol, what):
    got = got.double().cpu()
    off = (got - want).abs()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    ok = bool((same | (off <= tol)).all())
    assert ok, (what, float((off - tol)[~same].max()))


def _check_32(new_p, new_m, new_v, p, g, m, v, h, dtype):
    wp, wm, wv = ref.adamw(p, g, m, v, h["lr"], h["betas"], h["eps"], h["weight_decay"], h["step"], h.get("grad_scale", 1.0))
    b1, b2 = h["betas"]
    gd = g.double() * h.get("grad_scale", 1.0)
    if new_m is not None:
        _near(new_m, wm, 4 * U * (b1 * m.double().abs() + (1 - b1) * gd.abs()) + 1e-45, "m")
        _near(new_v, wv, 6 * U * wv + 1e-45, "v")
    t = h["step"] + 1
    room = 4 * U * (b1 * m.double().abs() + (1 - b1) * gd.abs())          # m's own error, as a step
    by = torch.sqrt(wv) / math.sqrt(1 - b2 ** t) + h["eps"]
    size = h["lr"] / (1 - b1 ** t)
    tol = 4 * U * p.double().abs() + 12 * U * size * wm.abs() / by + size * room / by + torch.finfo(dtype).eps / 2 * wp.abs()
    _near(new_p, wp, tol + (2.0 ** -25 if dtype == torch.float16 else 1e-45), "p")


HYPER = [dict(lr=1e-2, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.1, step=0), dict(lr=3e-3, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.0, step=41, grad_scale=0.25),
         dict(lr=1e-3, betas=(0.0, 0.0), eps=1e-3, weight_decay=0.01, step=3)]


@pytest.mark.parametrize("shift", [0, 1, 4])
@pytest.mark.parametrize("pt,gt,master", KINDS)
def test_steps_with_32_bit_states(slaq, pt, gt, master, shift):
    gen = torch.Generator().manual_seed(7 + shift)
    p, g = _cut(SIZES, pt, gen, 0.5, shift), _cut(SIZES, gt, gen, 0.1, shift)
    m = _cut(SIZES, torch.float32, gen, 0.05, shift)
    v = [x.square() for x in _cut(SIZES, torch.float32, gen, 0.05, shift)]
    masters = _cut(SIZES, torch.float32, gen, 0.5, shift) if master else None
    group_of = [k % 3 for k in range(len(SIZES))]
    plan = slaq.AdamW(p, g, group_of, HYPER, masters=masters, exp_avg=m, exp_avg_sq=v)
    for extra in range(3):
        old = [[x.cpu().clone() for x in xs] for xs in (masters or p, g, m, v)]
        plan.step()
        for k in range(len(SIZES)):
            h = dict(HYPER[group_of[k]])
            h["step"] += extra
            _check_32((masters or p)[k], m[k], v[k], *(xs[k] for xs in old), h, torch.float32 if master else pt)
            if master:
                assert torch.equal(p[k], masters[k].to(pt))
    np.testing.assert_array_equal(plan.get_steps(), [h["step"] + 3 for h in HYPER])


def _codes(x):
    """Nearest e4m3 values of x (|x| <= 448), as float64."""
    return x.float().to(torch.float8_e4m3fn).double()


@pytest.mark.parametrize("shift", [0, 1, 8])
@pytest.mark.parametrize("pt,gt,master", KINDS)
def test_steps_with_8_bit_states(slaq, pt, gt, master, shift):
    gen = torch.Generator().manual_seed(11 + shift)
    p, g = _cut(SIZES, pt, gen, 0.5, shift), _cut(SIZES, gt, gen, 0.1, shift)
    for x in g:
        x *= torch.exp(2 * torch.randn(x.shape, generator=gen)).to(gt).cuda()
    masters = _cut(SIZES, torch.float32, gen, 0.5, shift) if master else None
    codes = [torch.zeros(sum(SIZES) + shift, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2)]
    at = np.cumsum([shift] + SIZES)
    m, v = ([c[a: a + n] for a, n in zip(at, SIZES)] for c in codes)
    plan = slaq.AdamW(p, g, [k % 3 for k in range(len(SIZES))], HYPER, state_bits=8, masters=masters, exp_avg=m, exp_avg_sq=v)

    def values(codes, scales):
        return [(c.float().cpu() * s.cpu().repeat_interleave(256)[: c.numel()]) for c, s in zip(codes, scales)]
    for extra in range(3):
        old_m, old_r = values(plan.exp_avg, plan.exp_avg_scale), values(plan.exp_avg_sq, plan.exp_avg_sq_scale)
        old_p, old_g = [[x.cpu().clone() for x in xs] for xs in (masters or p, g)]
        plan.step()
        new_m, new_r = values(plan.exp_avg, plan.exp_avg_scale), values(plan.exp_avg_sq, plan.exp_avg_sq_scale)
        for k in range(len(SIZES)):
            h = dict(HYPER[k % 3])
            h["step"] += extra
            old_v = old_r[k] * old_r[k]
            _check_32((masters or p)[k], None, None, old_p[k], old_g[k], old_m[k], old_v, h, torch.float32 if master else pt)
            _, wm, wv = ref.adamw(old_p[k], old_g[k], old_m[k], old_v, h["lr"], h["betas"], h["eps"], h["weight_decay"], h["step"], h.get("grad_scale", 1.0))
            # e4m3 is spaced by 2^-9 below 2^-6: off by 2^-10 of the scale.  A root r in (0, 2^-10 s) becomes 2^-9 s instead of
            # 0 and is off by 2^-9 s - r < 2^-9 s.
            for got, want, scale, low in ((new_m[k], wm, plan.exp_avg_scale[k], 2.0 ** -10), (new_r[k], torch.sqrt(wv), plan.exp_avg_sq_scale[k], 2.0 ** -9)):
                s = scale.double().cpu().repeat_interleave(256)[: got.numel()]
                _near(got, want, (2.0 ** -4 + 1e-5) * want.abs() + low * s * (1 + 1e-5), "state")
            lost = (torch.sqrt(wv) > 0) & (new_r[k] == 0)
            assert not bool(lost.any())
            if master:
                assert torch.equal(p[k], masters[k].to(pt))


def test_a_block_is_rounded_as_e4m3_is(slaq):
    """With b1 = b2 = 0 the states are the gradients themselves: their codes follow from the type's own rounding.
    A scale is the largest x (1 / 448), a code the value x ((1 / largest) x 448), as the header says, all in 32 bits."""
    per = torch.tensor(1.0) / torch.tensor(448.0)
    g = torch.cat([torch.linspace(-3, 3, 256), torch.logspace(-8, 0, 256), torch.zeros(256), torch.full((100,), 1e-38)]).cuda()
    p = torch.zeros_like(g)
    plan = slaq.AdamW([p], [g], groups=[dict(betas=(0.0, 0.0))], state_bits=8)
    plan.step()
    for lo in range(0, g.numel(), 256):
        x = g[lo: lo + 256].cpu()
        most, b = x.abs().max(), lo // 256
        kept = most >= 2.0 ** -100
        inv = torch.tensor(1.0) / most * torch.tensor(448.0) if kept else torch.tensor(0.0)
        assert float(plan.exp_avg_scale[0][b]) == (float(most * per) if kept else 0.0)
        assert torch.equal(plan.exp_avg[0][lo: lo + 256].cpu().float(), (x * inv).to(torch.float8_e4m3fn).float())
        r = torch.sqrt(x * x)
        most = r.max()
        inv = torch.tensor(1.0) / most * torch.tensor(448.0) if kept else torch.tensor(0.0)
        want = torch.where((r > 0) & bool(kept), (r * inv).clamp_min(2.0 ** -9), r * inv).to(torch.float8_e4m3fn).float()
        assert torch.equal(plan.exp_avg_sq[0][lo: lo + 256].cpu().float(), want)


@pytest.mark.parametrize("bits", [8, 32])
def test_groups_without_cores_stay_as_they_are(slaq, bits):
    gen = torch.Generator().manual_seed(3)
    sizes = [300, 1000, 5, 2049]
    p, g = _cut(sizes, torch.bfloat16, gen, 0.5), _cut(sizes, torch.bfloat16, gen, 0.1)
    plan = slaq.AdamW(p, g, [0, 1, 1, 2], [{}, {"step": 5}, {}], state_bits=bits)
    every = lambda: [x.clone() for xs in (plan.params, plan.exp_avg, plan.exp_avg_sq) for x in xs]   # noqa: E731
    before = every()
    plan.step(torch.tensor([0, 3, -1], dtype=torch.int32, device="cuda"))
    after = every()
    for k, (a, b) in enumerate(zip(before, after)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)) == (k % 4 in (0, 3))
    np.testing.assert_array_equal(plan.get_steps(), [0, 6, 0])
    plan.set_group(0, lr=0.5)
    plan.set_group(1, step=100)
    plan.step()
    np.testing.assert_array_equal(plan.get_steps(), [1, 101, 1])
    torch.testing.assert_close(plan.params[0].float(), before[0].float() - 0.5 * torch.sign(g[0].float()) - 0.5 * 0.01 * before[0].float(), rtol=2 ** -7, atol=1e-5)


@pytest.mark.parametrize("bits", [8, 32])
def test_what_is_not_finite_stays_in_its_element(slaq, bits):
    p, g = torch.ones(600, device="cuda"), torch.full((600,), 0.1, device="cuda")
    g[3], g[300], g[599] = math.nan, math.inf, -math.inf
    plan = slaq.AdamW([p], [g], state_bits=bits)
    for _ in range(2):
        plan.step()
        bad = torch.zeros(600, dtype=torch.bool, device="cuda")
        bad[[3, 300, 599]] = True
        assert torch.equal(~p.isfinite(), bad)
        if bits == 8:
            assert torch.equal(plan.exp_avg_sq[0].float().isnan(), bad) and torch.equal(plan.exp_avg[0].float().isnan(), bad)
            assert bool(plan.exp_avg_scale[0].isfinite().all())


@pytest.mark.parametrize("bits", [8, 32])
def test_replayed_steps_are_the_same_as_called_ones(slaq, bits):
    gen = torch.Generator().manual_seed(5)
    sizes = [70_000, 33, 512]
    start, g = _cut(sizes, torch.float32, gen, 0.5), _cut(sizes, torch.float32, gen, 0.1)
    on = torch.tensor([1, 0], dtype=torch.int32, device="cuda")
    results = []
    for captured in (False, True):
        p = [x.clone() for x in start]
        plan = slaq.AdamW(p, g, [0, 1, 0], [{"lr": 1e-2}, {}], state_bits=bits)
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                plan.step(on)
            np.testing.assert_array_equal(plan.get_steps(), [0, 0])
        for k in range(4):
            if k == 2:
                plan.set_group(0, lr=5e-3)
            graph.replay() if captured else plan.step(on)
        np.testing.assert_array_equal(plan.get_steps(), [4, 0])
        results.append(p)
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_other_gradients_and_another_stream(slaq):
    gen = torch.Generator().manual_seed(5)
    p, g, g2 = (_cut([1000, 10], torch.float32, gen, 0.5) for _ in range(3))
    q = [x.clone() for x in p]
    a, b = slaq.AdamW(p, g), slaq.AdamW(q, g2)
    a.set_grads(g2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a.step(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    b.step()
    assert all(torch.equal(x, y) for x, y in zip(p, q))


@pytest.mark.parametrize("pt,shift", [(torch.bfloat16, 0), (torch.bfloat16, 3), (torch.float32, 0)])
@pytest.mark.parametrize("bits", [8, 32])
def test_a_large_plan_is_the_sum_of_small_ones(slaq, bits, pt, shift):
    """Blocks do not know of one another: tensors cut at block boundaries into plans of their own give the same bits."""
    gen = torch.Generator().manual_seed(13)
    sizes = [5_000_003, 700, 256 * 32, 900_001, 1, 256 * 33 - 1]
    p, g = _cut(sizes, pt, gen, 0.5, shift), _cut(sizes, pt, gen, 0.1, shift)
    blocks = lambda n: -(-n // 256)   # noqa: E731
    state = torch.float8_e4m3fn if bits == 8 else torch.float32
    make = lambda xs: (dict(exp_avg=[torch.zeros(x.numel(), device="cuda").to(state) for x in xs], exp_avg_sq=[torch.zeros(x.numel(), device="cuda").to(state) for x in xs])   # noqa: E731
                       | (dict(exp_avg_scale=[torch.zeros(blocks(x.numel()), device="cuda") for x in xs], exp_avg_sq_scale=[torch.zeros(blocks(x.numel()), device="cuda") for x in xs]) if bits == 8 else {}))
    whole, q = make(p), [x.clone() for x in p]
    plan = slaq.AdamW(p, g, state_bits=bits, **whole)
    pieces = make(q)
    plans = []
    for k, n in enumerate(sizes):
        for lo in range(0, n, 256 * 4000):
            hi = min(n, lo + 256 * 4000)
            part = {name: [v[k][lo // 256: blocks(hi)] if "scale" in name else v[k][lo:hi]] for name, v in pieces.items()}
            plans.append(slaq.AdamW([q[k][lo:hi]], [g[k][lo:hi]], state_bits=bits, **part))
    for _ in range(3):
        plan.step()
        for x in plans:
            x.step()
    for a, b in zip(p, q):
        assert torch.equal(a, b)
    for name in whole:
        for a, b in zip(whole[name], pieces[name]):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), name


def test_many_small_tensors(slaq):
    gen = torch.Generator().manual_seed(9)
    sizes = [1 + k % 40 for k in range(5000)]
    p, g = _cut(sizes, torch.float32, gen, 0.5), _cut(sizes, torch.float32, gen, 0.1)
    before = torch.cat(p).cpu()
    hyper = [dict(lr=1e-3 * (1 + k % 5), betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, step=k % 50) for k in range(1000)]
    plan = slaq.AdamW(p, g, [k // 5 for k in range(5000)], hyper)
    plan.step()
    at = 0
    for k, n in enumerate(sizes[:400]):
        z = torch.zeros(n)
        _check_32(p[k], plan.exp_avg[k], plan.exp_avg_sq[k], before[at: at + n], g[k].cpu(), z, z, hyper[k // 5], torch.float32)
        at += n


@pytest.mark.parametrize("given", [False, True])
def test_memory_of_the_librarys_own_or_of_the_caller(slaq, given):
    import ctypes

    from paper_1802_04819_b200.training import _group, _Tensor
    lib = slaq.load_library()
    p, g, m, v = (torch.full((700,), x, device="cuda") for x in (1.0, 0.5, 0.0, 0.0))
    table, groups, numels = (_Tensor * 1)(), (type(_group()) * 1)(_group(lr=0.25, weight_decay=0.0)), (ctypes.c_int64 * 1)(700)
    for name, t in (("param", p), ("grad", g), ("exp_avg", m), ("exp_avg_sq", v)):
        setattr(table[0], name, t.data_ptr())
    table[0].n = 700
    need = lib.slaq_adamw_workspace_bytes(1, ctypes.addressof(numels), 1)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    h = ctypes.c_void_p()
    assert lib.slaq_adamw_create(ws.data_ptr(), need - 1, 1, table, 1, groups, 0, 0, 32, None, ctypes.byref(h)) == -4 and not h.value
    assert lib.slaq_adamw_create(ws.data_ptr() if given else None, need if given else 0, 1, table, 1, groups, 0, 0, 32, None, ctypes.byref(h)) == 0
    assert lib.slaq_adamw_step(h, None, None) == 0
    torch.cuda.synchronize()
    torch.testing.assert_close(p, torch.full_like(p, 0.75), rtol=1e-6, atol=0)
    assert lib.slaq_adamw_destroy(h) == 0


def test_a_plan_that_is_dropped_while_another_stream_steps(slaq):
    """Its memory is not given to anybody before that stream has passed the steps."""
    side = torch.cuda.Stream()
    n = 3_000_000
    p, g = torch.ones(n, device="cuda"), torch.ones(n, device="cuda")
    torch.cuda.synchronize()
    plan = slaq.AdamW([p], [g], groups=[dict(lr=0.01, weight_decay=0.0)])
    torch.cuda.synchronize()
    for _ in range(20):
        plan.step(stream=side)
    m, v = plan.exp_avg, plan.exp_avg_sq           # the states are the caller's to keep
    del plan
    junk = [torch.full((300_000,), 255, dtype=torch.uint8, device="cuda") for _ in range(20)]
    torch.cuda.synchronize()
    torch.testing.assert_close(p, torch.full_like(p, 0.8), rtol=0, atol=1e-4)
    del junk, m, v


def test_refusals(slaq):
    flat, g = torch.zeros(100, device="cuda"), torch.zeros(50, device="cuda")
    a, b = flat[:50], flat[50:]
    for call in (lambda: slaq.AdamW([a, a], [g, g]), lambda: slaq.AdamW([a, flat[40:90]], [g, g]), lambda: slaq.AdamW([a], [a]), lambda: slaq.AdamW([], []),
                 lambda: slaq.AdamW([a], [g], [1]), lambda: slaq.AdamW([a], [g], [-1]), lambda: slaq.AdamW([a], [g], groups=[]),
                 lambda: slaq.AdamW([a], [g], groups=[{"betas": (1.0, 0.9)}]), lambda: slaq.AdamW([a], [g], groups=[{"betas": (0.9, -0.1)}]),
                 lambda: slaq.AdamW([a], [g], groups=[{"lr": -1.0}]), lambda: slaq.AdamW([a], [g], groups=[{"eps": math.nan}]),
                 lambda: slaq.AdamW([a], [g], groups=[{"step": -1}]), lambda: slaq.AdamW([a], [g[:49]]), lambda: slaq.AdamW([a], [g.double()]),
                 lambda: slaq.AdamW([a], [g], state_bits=16), lambda: slaq.AdamW([a], [g.half()]), lambda: slaq.AdamW([a.cpu()], [g]),
                 lambda: slaq.AdamW([a, b], [g, g], exp_avg=[torch.zeros(50, device="cuda")] * 2),
                 lambda: slaq.AdamW([flat.view(10, 10).t()], [g]), lambda: slaq.AdamW([a], [g], masters=[a])):
        with pytest.raises(slaq.SlaqError) as e:
            call()
        assert e.value.code == -1
    plan = slaq.AdamW([a, b], [g, g])
    for call, code in ((lambda: plan.step(torch.ones(2, dtype=torch.int32, device="cuda")), -1), (lambda: plan.set_group(1, lr=1.0), -2),
                       (lambda: plan.set_group(0, lr=-1.0), -1), (lambda: plan.set_grads([g]), -1), (lambda: plan.set_grads([a, g]), -1)):
        with pytest.raises(slaq.SlaqError) as e:
            call()
        assert e.value.code == code
