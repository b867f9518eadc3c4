"""AdamW at the ends of what its groups may hold."""

import pytest
import torch

import token_rows as ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def slaq():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_1802_04819_b200 as mod
    mod.build()
    return mod


@pytest.mark.parametrize("eps", [2.0 ** -126, 1.2e-38, 1e-30])
@pytest.mark.parametrize("bits", [8, 32])
def test_the_smallest_epsilons(slaq, bits, eps):
    """Where gradient and states are 0 the step is 0 / eps = 0.  Elsewhere eps is nothing beside the root (at least 1e-18 here), so the
    first step is lr times the gradient's sign, off by the 12 roundings of the step (see test_gpu_adamw) and the weight's own."""
    g = torch.zeros(1000, device="cuda")
    g[3::7], g[700] = 0.01, 1e-15
    p = torch.full_like(g, 0.5)
    plan = slaq.AdamW([p], [g], groups=[dict(lr=1e-2, eps=eps, weight_decay=0.0)], state_bits=bits)
    plan.step()
    z = torch.zeros(1000)
    want, _, _ = ref.adamw(torch.full((1000,), 0.5), g.cpu(), z, z, 1e-2, (0.9, 0.999), eps, 0.0, 0)
    off = (p.double().cpu() - want).abs()
    assert not p.isnan().any() and float(off.max()) <= 20 * U * 1e-2 + U
    assert bool((p[g == 0] == 0.5).all())


@pytest.mark.parametrize("eps", [1e-40, 2.0 ** -127])
def test_smaller_ones_are_refused(slaq, eps):
    p, g = torch.zeros(10, device="cuda"), torch.zeros(10, device="cuda")
    with pytest.raises(slaq.SlaqError):
        slaq.AdamW([p], [g], groups=[dict(eps=eps)])
    plan = slaq.AdamW([p], [g])
    with pytest.raises(slaq.SlaqError):
        plan.set_group(0, eps=eps)
    plan.step()
    assert not p.any()
