"""Limits of norms that are no limits."""

import math

import pytest
import torch

from test_gpu_grad_norms import slaq  # noqa: F401

pytestmark = pytest.mark.gpu


def test_a_negative_limit_leaves_its_group_alone(slaq):  # noqa: F811
    grads = [torch.full((100,), 0.5, device="cuda") for _ in range(6)]
    grads[3].zero_()
    limits = torch.tensor([-1.0, 2.0, -math.inf, -1e-30, -0.0, math.inf], device="cuda")
    plan = slaq.GradNorms(grads, range(6))
    norm, factor = plan.measure(limits)
    assert norm.tolist() == [5.0, 5.0, 5.0, 0.0, 5.0, 5.0]
    assert [math.isnan(f) for f in factor.tolist()] == [True, False, True, True, False, False]
    assert float(factor[1]) == pytest.approx(0.4, rel=1e-6) and factor[4:].tolist() == [0.0, 1.0]
    weights = [torch.ones(100, device="cuda") for _ in range(6)]
    adamw = slaq.AdamW(weights, grads, range(6), [dict(lr=0.1)] * 6)
    adamw.step(factors=factor)
    assert adamw.get_steps().tolist() == [0, 1, 0, 0, 1, 1]
    assert all(bool((weights[k] == 1).all()) for k in (0, 2, 3))
    plan.apply(factor)
    assert [float(g[0]) for g in grads] == pytest.approx([0.5, 0.2, 0.5, 0.0, 0.0, 0.5])
