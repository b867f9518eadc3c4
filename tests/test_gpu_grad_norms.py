"""Norms of groups of gradients and clipping, against 64 bits.

Tolerances (u = 2^-24): a lane's squares go through at most 8 fused additions and 3 joins in 32 bits, 11u of a sum of positive terms, hence 5.5u of its
root; what follows is in 64 bits and rounded once: 7u of a norm.  A factor is a quotient of that norm before its rounding: 7u as well.
Products with a factor are rounded once: exactly the formula's."""

import math

import numpy as np
import pytest
import torch

from test_gpu_adamw import HYPER, SIZES, _check_32, _cut

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def slaq():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_1802_04819_b200 as mod
    mod.build()
    return mod


def _norms(grads, group_of, n_groups, scale=1.0):
    out = np.zeros(n_groups)
    for g, k in zip(grads, group_of):
        out[k] += float(g.double().square().sum())
    return abs(scale) * np.sqrt(out)


def _check(got, want, rel=7 * U):
    np.testing.assert_allclose(got.double().cpu().numpy(), want, rtol=rel, atol=0)


@pytest.mark.parametrize("shift", [0, 1, 3, 8])
@pytest.mark.parametrize("dtype", TYPES)
def test_norms_and_factors(slaq, dtype, shift):
    gen = torch.Generator().manual_seed(3 + shift)
    sizes = SIZES + [70_001, 9000]
    grads = _cut(sizes, dtype, gen, 0.1, shift)
    group_of = [k % 4 for k in range(len(sizes))]
    plan = slaq.GradNorms(grads, group_of, n_groups=5)         # the last group has no tensor
    want = _norms(grads, group_of, 5)
    most = float(np.median(want))
    norm, factor = plan.measure(most)
    _check(norm, want)
    clipped = want > most
    assert 0 < clipped.sum() < 5
    _check(factor, np.where(clipped, most / np.maximum(want, 1e-30), 1.0))
    assert factor[4] == 1 and norm[4] == 0
    norm, factor = plan.measure(scale=-0.3)                    # no largest norm
    _check(norm, 0.3 * want)
    assert bool((factor == 1).all())


@pytest.mark.parametrize("groups", [1, 2, 7, 8, 9, 300])
def test_groups_in_any_order_and_of_any_number(slaq, groups):
    gen = torch.Generator().manual_seed(groups)
    sizes = [int(n) for n in torch.randint(1, 20_000, (max(20, groups + 5),), generator=gen)]
    grads = _cut(sizes, torch.bfloat16, gen, 1.0)
    group_of = torch.randint(groups, (len(sizes),), generator=gen).tolist()
    norm, _ = slaq.GradNorms(grads, group_of, n_groups=groups).measure(1.0)
    _check(norm, _norms(grads, group_of, groups))


def test_tensors_of_several_types_in_one_group(slaq):
    gen = torch.Generator().manual_seed(1)
    grads = [t for dtype in TYPES for t in _cut([1, 1000, 33_333], dtype, gen, 0.5, 1)]
    norm, factor = slaq.GradNorms(grads).measure(2.0)
    want = _norms(grads, [0] * len(grads), 1)
    _check(norm, want)
    _check(factor, 2.0 / want)


def test_a_tensor_of_many_units_for_every_warp(slaq):
    gen = torch.Generator(device="cuda").manual_seed(1)
    big, small = torch.randn(80_000_003, generator=gen, device="cuda"), torch.randn(5, generator=gen, device="cuda")
    for dtype in (torch.float32, torch.bfloat16):
        grads = [big.to(dtype)[1:], small.to(dtype), big.to(dtype)[: 30_000_000] * 0.5]
        norm, _ = slaq.GradNorms(grads, [0, 1, 0]).measure()
        _check(norm, _norms(grads, [0, 1, 0], 2))


@pytest.mark.parametrize("dtype,size", [(torch.float32, 1e-30), (torch.float32, 1e-42), (torch.float32, 1e25), (torch.float32, 3e38), (torch.bfloat16, 1e-38),
                                        (torch.bfloat16, 2e38), (torch.float16, 6e-8), (torch.float16, 6e4), (torch.float32, 2.0 ** -51)])
def test_squares_that_32_bits_do_not_hold(slaq, dtype, size):
    x = torch.full((5000,), size, dtype=dtype, device="cuda")
    x[::3] *= -0.5
    x[4000:] = 0
    grads = [x, x[:3].clone()]
    norm, factor = slaq.GradNorms(grads, [0, 1]).measure(size)
    want = _norms(grads, [0, 1], 2)
    # above 32 bits a norm is infinite, but not its factor; below 2^-126 a norm is a multiple of 2^-149
    big = want > float(np.finfo(np.float32).max)
    got = norm.double().cpu().numpy()
    assert np.isinf(got[big]).all()
    np.testing.assert_allclose(got[~big], want[~big], rtol=7 * U, atol=2.0 ** -150)
    _check(factor, np.minimum(size / want, 1.0))


def test_zeros_and_empty_tensors(slaq):
    grads = [torch.zeros(3000, device="cuda"), torch.full((3000,), -0.0, device="cuda", dtype=torch.bfloat16), torch.empty(0, device="cuda")]
    for most in (0.0, 1.0):
        norm, factor = slaq.GradNorms(grads, [0, 1, 2]).measure(most)
        assert norm.tolist() == [0, 0, 0] and factor.tolist() == [1, 1, 1]
    norm, factor = slaq.GradNorms([torch.ones(7, device="cuda")]).measure(0.0)
    assert factor.tolist() == [0.0]


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("at", [0, 7, 1500, 2999])
def test_what_is_not_finite_stays_in_its_group(slaq, bad, at):
    for dtype in TYPES:
        x = torch.ones(3000, device="cuda", dtype=dtype)
        x[at] = bad
        ones = torch.ones(100, device="cuda")
        plan = slaq.GradNorms([x, ones], [0, 1])
        norm, factor = plan.measure(5.0)
        assert (math.isnan(norm[0]) if math.isnan(bad) else norm[0] == math.inf) and math.isnan(factor[0])
        assert norm[1] == 10 and factor[1] == 0.5
        old = x.clone()
        plan.apply(factor)
        assert torch.equal(x.nan_to_num(5), old.nan_to_num(5)) and bool((ones == 0.5).all())


def test_idle_groups_are_not_read_and_limits_per_group(slaq):
    grads = [torch.full((2000,), 0.1 * (k + 1), device="cuda") for k in range(5)]
    active = torch.tensor([1, 0, 4, -2, 1], dtype=torch.int32, device="cuda")
    mosts = torch.tensor([1.0, 1.0, 1e9, 1.0, math.nan], device="cuda")
    old = [g.clone() for g in grads]
    plan = slaq.GradNorms(grads, range(5))
    norm, factor = plan.measure(mosts, active=active)
    want = _norms(grads, range(5), 5)
    _check(norm, want * np.array([1, 0, 1, 0, 1]))
    assert factor[1:4].tolist() == [1.0, 1.0, 1.0] and math.isnan(factor[4])
    _check(factor[:1], 1.0 / want[:1])
    plan.apply(torch.full((5,), 0.5, device="cuda"), active=active)
    for k, (g, was) in enumerate(zip(grads, old)):
        assert torch.equal(g, was * 0.5 if active[k] > 0 else was)


@pytest.mark.parametrize("to,shift", [(None, 0), (0, 0), (1, 0), (0, 3), (2, 2), (5, 1)])
@pytest.mark.parametrize("dtype", TYPES)
def test_products_with_factors(slaq, dtype, to, shift):
    gen = torch.Generator().manual_seed(shift)
    sizes = SIZES + [30_000]
    grads = _cut(sizes, dtype, gen, 0.1, shift)
    out = None if to is None else _cut(sizes, dtype, gen, 1.0, to)
    group_of = [k % 4 for k in range(len(sizes))]
    factor = torch.tensor([0.3, 1.0, math.nan, 0.0], device="cuda")
    old, held = [g.clone() for g in grads], [x.clone() for x in (out or grads)]
    plan = slaq.GradNorms(grads, group_of, out=out)
    plan.apply(factor)
    for k, (g, was, had, got) in enumerate(zip(grads, old, held, out or grads)):
        f = float(factor[group_of[k]])
        want = had if math.isnan(f) else (was.float() * factor[group_of[k]]).to(dtype)
        assert torch.equal(got, want), k
        if out is not None:
            assert torch.equal(g, was)


def test_nothing_beside_the_tensors_is_written(slaq):
    for dtype in TYPES:
        buffer = torch.full((4000,), 2.0, dtype=dtype, device="cuda")
        tensors = [buffer[a:b] for a, b in ((1, 2), (5, 17), (18, 1900), (1901, 3999))]
        inside = torch.zeros(4000, dtype=torch.bool, device="cuda")
        for a, b in ((1, 2), (5, 17), (18, 1900), (1901, 3999)):
            inside[a:b] = True
        slaq.GradNorms(tensors).apply(torch.tensor([0.5], device="cuda"))
        assert torch.equal(buffer, torch.where(inside, 1.0, 2.0).to(dtype))


@pytest.mark.parametrize("state_bits", [32, 8])
@pytest.mark.parametrize("dtype,master", [(torch.float32, False), (torch.bfloat16, False), (torch.bfloat16, True)])
def test_a_step_takes_the_factors(slaq, dtype, master, state_bits):
    """As a step over gradients multiplied beforehand, which for powers of two have the same bits; groups whose factor is not finite, or that
    have none, are left as they are, their counts too."""
    gen = torch.Generator().manual_seed(5)
    factors = torch.tensor([0.5, 2.0, math.nan, math.inf, 0.25], device="cuda")
    for factor_of, of in ((None, [0, 1, 2, 3, 4]), ([1, 4, 0, 2, 5], [1, 4, 0, 2, 5]), ([-1, 0, 0, 0, 1 << 30], [-1, 0, 0, 0, 1 << 30])):
        p, g = _cut(SIZES, dtype, gen, 0.5), _cut(SIZES, dtype, gen, 0.1)
        masters = [x.float() for x in p] if master else None
        group_of, n = [k % 5 for k in range(len(SIZES))], len(SIZES)
        kept = [0 <= f < 5 and math.isfinite(factors[f]) for f in of]
        groups = [dict(HYPER[k % 3], grad_scale=0.5) for k in range(5)]
        make = lambda p, g, m: slaq.AdamW(p, g, group_of, groups, state_bits=state_bits, masters=m)   # noqa: E731
        other = [x.clone() for x in p], [x * float(factors[of[k]]) if kept[k] else x.clone() for x, k in zip(g, group_of)], masters and [x.clone() for x in masters]
        a, b = make(p, g, masters), make(*other)
        mapped = None if factor_of is None else torch.tensor(factor_of, dtype=torch.int32, device="cuda")
        active = torch.tensor(kept, device="cuda").int()
        for _ in range(2):
            a.step(factors=factors, factor_of=mapped)
            b.step(active)
        for name in ("params", "masters", "exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale"):
            for x, y in zip(getattr(a, name) or (), getattr(b, name) or ()):
                same = x.view(torch.uint8), y.view(torch.uint8)
                assert torch.equal(*same), name
        np.testing.assert_array_equal(a.get_steps(), b.get_steps())
        assert len(p) == n


def test_a_clipped_step_against_the_formula(slaq):
    gen = torch.Generator().manual_seed(9)
    p, g = _cut(SIZES, torch.float32, gen, 0.5), _cut(SIZES, torch.float32, gen, 0.1)
    group_of = [k % 3 for k in range(len(SIZES))]
    groups = [{k: v for k, v in h.items() if k != "grad_scale"} for h in HYPER]
    plan, norms = slaq.AdamW(p, g, group_of, groups), slaq.GradNorms(g, group_of)
    old = [x.cpu().clone() for x in p]
    norm, factor = norms.measure(1.0)
    assert bool((factor < 1).any())
    plan.step(factors=factor)
    for k in range(len(SIZES)):
        h = dict(groups[group_of[k]], grad_scale=float(factor[group_of[k]]))
        zero = torch.zeros(SIZES[k])
        _check_32(p[k], plan.exp_avg[k], plan.exp_avg_sq[k], old[k], g[k].cpu(), zero, zero, h, torch.float32)


def test_other_gradients_and_the_same_sums_every_time(slaq):
    gen = torch.Generator().manual_seed(2)
    sizes = [100_000, 33, 250_001]
    a, b = _cut(sizes, torch.bfloat16, gen, 1.0), _cut(sizes, torch.bfloat16, gen, 2.0, 1)
    plan = slaq.GradNorms(a)
    first = plan.measure(1.0)
    for _ in range(20):
        again = plan.measure(1.0)
        assert torch.equal(first.norm, again.norm) and torch.equal(first.factor, again.factor)
    plan.set_grads(b)
    _check(plan.measure(1.0).norm, _norms(b, [0] * 3, 1))
    plan.apply(torch.tensor([0.5], device="cuda"))       # in place: the new ones
    _check(plan.measure(1.0).norm, _norms(b, [0] * 3, 1))


def test_captured_and_replayed_on_other_streams(slaq):
    gen = torch.Generator().manual_seed(4)
    grads = _cut([5000, 70_000], torch.float32, gen, 1.0)
    plan = slaq.GradNorms(grads, [0, 1])
    norm, factor = torch.empty(2, device="cuda"), torch.empty(2, device="cuda")
    plan.measure(1.0, norm=norm, factor=factor)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.measure(3.0, norm=norm, factor=factor)
        plan.apply(factor)
    for size in (1.0, 4.0):
        for g in grads:
            g.copy_(torch.randn(g.shape, generator=gen) * size)
        want = _norms(grads, [0, 1], 2)
        graph.replay()
        _check(norm, want)
        _check(plan.measure().norm, np.minimum(want, 3.0), 9 * U)       # one more rounding each: of the factor and of the products
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    on_side = plan.measure(1.0, stream=side)
    raw = plan.measure(1.0, stream=side.cuda_stream)
    side.synchronize()
    want = _norms(grads, [0, 1], 2)
    _check(on_side.norm, want)
    _check(raw.norm, want)


def test_what_is_written_counts_as_changed(slaq):
    g, o = torch.ones(10, device="cuda"), torch.ones(10, device="cuda")
    plan = slaq.GradNorms([g])
    v = g._version
    plan.measure(1.0)
    assert g._version == v
    plan.apply(torch.ones(1, device="cuda"))
    assert g._version == v + 1
    flat = torch.ones(30, device="cuda")
    parts, v = [flat[:10], flat[10:]], flat._version
    slaq.GradNorms(parts).apply(torch.ones(1, device="cuda"))
    assert flat._version == parts[0]._version == parts[1]._version == v + 1
    given = torch.empty(1, device="cuda")
    v = given._version
    slaq.GradNorms([g], out=[o]).measure(1.0, norm=given)
    assert given._version == v + 1


def test_refusals_from_python(slaq):
    x = torch.ones(100, device="cuda")
    for bad in (lambda: slaq.GradNorms([]), lambda: slaq.GradNorms([torch.ones(3)]), lambda: slaq.GradNorms([x.double()]),
                lambda: slaq.GradNorms([x, x]), lambda: slaq.GradNorms([x[:60], x[50:]]), lambda: slaq.GradNorms([x], [1], n_groups=1),
                lambda: slaq.GradNorms([x], [-1]), lambda: slaq.GradNorms([x], [0, 0]), lambda: slaq.GradNorms([x[::2]]),
                lambda: slaq.GradNorms([x], out=[x[:50]]), lambda: slaq.GradNorms([x], out=[x.bfloat16()]), lambda: slaq.GradNorms([x[:50]], out=[x[10:60]]),
                lambda: slaq.GradNorms([x], out=[])):
        with pytest.raises(slaq.SlaqError):
            bad()
    plan = slaq.GradNorms([x])
    two = torch.ones(2, device="cuda")
    for bad in (lambda: plan.measure(-1.0), lambda: plan.measure(math.nan), lambda: plan.measure(two), lambda: plan.measure(1.0, active=two),
                lambda: plan.measure(1.0, scale=math.inf), lambda: plan.measure(1.0, norm=two), lambda: plan.apply(two), lambda: plan.apply(None),
                lambda: plan.set_grads([two]), lambda: plan.set_grads([]), lambda: plan.apply(torch.ones(1))):
        with pytest.raises(slaq.SlaqError):
            bad()
    adamw = slaq.AdamW([torch.ones(3, device="cuda")], [torch.ones(3, device="cuda")])
    for bad in (lambda: adamw.step(factors=two), lambda: adamw.step(factor_of=torch.zeros(1, dtype=torch.int32, device="cuda")),
                lambda: adamw.step(factors=two, factor_of=two), lambda: adamw.step(factors=two[:0], factor_of=torch.zeros(1, dtype=torch.int32, device="cuda"))):
        with pytest.raises(slaq.SlaqError):
            bad()
