"""Draws from the largest vocabulary, from rows beyond 2^31 elements, and norms of tensors beyond 2^31 elements."""

import numpy as np
import pytest
import torch

import sampling

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def slaq():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_1802_04819_b200 as mod
    mod.build()
    return mod


def _check(slaq, x, u, **numbers):
    got = slaq.sample_tokens(x, u, **numbers)
    for r in range(x.shape[0]):
        want = sampling.draw(x[r].double().cpu().numpy(), float(u[r]), numbers.get("temperature", 1.0), numbers.get("top_k", 0), numbers.get("top_p", 1.0), numbers.get("min_p", 0.0))
        assert want[4] > 2.0 ** -45 and int(got.token[r]) == want[0]
        assert got.kept is None or int(got.kept[r]) == want[3]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_largest_vocabulary(slaq, dtype):
    g = torch.Generator(device="cuda").manual_seed(1)
    x = (torch.randn(3, 1 << 22, generator=g, device="cuda") * 2).to(dtype)
    x[0, 4_000_001] = 30.0
    u = torch.rand(3, generator=g, device="cuda")
    for numbers in (dict(), dict(top_k=40), dict(top_p=0.9), dict(top_k=100_000, top_p=0.5), dict(min_p=0.01)):
        _check(slaq, x, u, **numbers)
    with pytest.raises(slaq.SlaqError):
        slaq.sample_tokens(torch.empty(1, (1 << 22) + 1, device="cuda"), u[:1])


def test_rows_beyond_2_to_the_31(slaq):
    rows, vocab = 40_000, 65_536
    x = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(2)
    u = torch.full((rows,), -1.0, device="cuda")
    last = slice(rows - 20, rows)
    x[last] = torch.randn(20, vocab, generator=g, device="cuda").bfloat16() * 3
    u[last] = torch.rand(20, generator=g, device="cuda")
    for numbers in (dict(), dict(top_k=30, top_p=0.9)):
        got = slaq.sample_tokens(x, u, **numbers)
        alone = slaq.sample_tokens(x[last].clone(), u[last].clone(), **numbers)
        assert torch.equal(got.token[last], alone.token) and bool((got.token[: rows - 20] == -1).all())
        _check(slaq, x[last], u[last], **numbers)


def test_tensors_beyond_2_to_the_31(slaq):
    n = (1 << 31) + 12_345
    x = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    x[-5:] = 3.0
    x[7] = 4.0
    y = torch.ones(3, device="cuda")
    plan = slaq.GradNorms([x, y], [0, 1])
    norm, factor = plan.measure(1.0)
    want = np.sqrt([5 * 9.0 + 16.0, 3.0])
    np.testing.assert_allclose(norm.double().cpu().numpy(), want, rtol=7 * 2.0 ** -24)
    plan.apply(torch.tensor([0.5, 1.0], device="cuda"))
    assert x[-5:].tolist() == [1.5] * 5 and x[7] == 2.0 and y.tolist() == [1.0] * 3
