"""Plans whose products go to a given tensor."""

import pytest
import torch

from test_gpu_grad_norms import slaq  # noqa: F401

pytestmark = pytest.mark.gpu


def test_a_given_output_stays_the_output(slaq):  # noqa: F811
    """.. also where it was the gradient itself."""
    a, b = torch.full((3000,), 2.0, device="cuda"), torch.full((3000,), 8.0, device="cuda")
    plan = slaq.GradNorms([a], out=[a])
    half = torch.full((1,), 0.5, device="cuda")
    plan.apply(half)
    assert bool((a == 1).all())
    plan.set_grads([b])
    versions = a._version, b._version
    plan.apply(half)
    assert bool((a == 4).all()) and bool((b == 8).all())
    assert (a._version, b._version) == (versions[0] + 1, versions[1])
