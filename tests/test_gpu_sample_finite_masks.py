"""Rows in which tokens are forbidden by large finite numbers, as ``masked_fill(mask, torch.finfo(dtype).min)`` does: their weights are 0 in 64 bits, and
nothing else about the row changes.  Tolerances are those of test_gpu_sample_tokens."""

import math

import pytest
import torch

from test_gpu_sample_tokens import _check, _rows, slaq  # noqa: F401

pytestmark = pytest.mark.gpu

# At temperature 1 exponents of 32 bits hold 2^127: a weight against a base of -3e9 or less may be anything.
VALUES = [("min", 1.0), (-1e30, 0.7), (-1e10, 1.0), (-1e9, 0.01), (-1e7, 1e-3)]
NUMBERS = [dict(), dict(top_p=1.0), dict(top_k=20), dict(top_p=0.9), dict(min_p=0.05), dict(top_p=0.8, min_p=0.01), dict(top_k=3000, top_p=0.95, min_p=0.001)]
SHARES = [0.0, 0.3, 0.9, 0.999, 1.0]


def _masked(rows, vocab, dtype, value, seed, height):
    """Row r: a share of SHARES, in turn scattered, in one run from the front, in one up to the end."""
    x, u = _rows(rows, vocab, dtype, seed, height=height, pad=5, first=3)
    g = torch.Generator().manual_seed(seed + 1)
    value = torch.finfo(dtype).min if value == "min" else value
    for r in range(rows):
        n = int(SHARES[r % len(SHARES)] * vocab)
        where = (torch.randperm(vocab, generator=g)[:n], torch.arange(n), torch.arange(vocab - n, vocab))[r // len(SHARES) % 3]
        x[r, where.cuda()] = value
    return x, u


@pytest.mark.parametrize("value,T", VALUES, ids=str)
@pytest.mark.parametrize("vocab", [20, 700, 1500, 5000, 130_001])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_finite_masks(slaq, dtype, vocab, value, T):  # noqa: F811
    for height, width in ((16.0, 1.0), (2.0, T)):             # peaked rows, and rows that keep much
        x, u = _masked(15, vocab, dtype, value, vocab, height * width)
        for numbers in NUMBERS if vocab < 100_000 or width == T else NUMBERS[3:5]:
            _check(slaq.sample_tokens(x, u, T, **numbers), x, u, T, **numbers)


@pytest.mark.parametrize("vocab", [1500, 5000, 20_000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_finite_masks_in_many_rows(slaq, dtype, vocab):  # noqa: F811
    x, u = _masked(305, vocab, dtype, "min", vocab, 12.0)
    for numbers in (dict(), dict(top_p=0.9), dict(top_k=1200, top_p=0.9)) if vocab < 20_000 else (dict(top_p=0.9),):
        _check(slaq.sample_tokens(x, u, **numbers), x, u, **numbers)


def test_a_log_probability_is_a_number_beside_finite_masks(slaq):  # noqa: F811
    """What a mask of either kind gives has the same bits."""
    x, u = _rows(40, 9000, torch.float32, 3, height=18.0)
    gone = torch.rand(40, 9000, generator=torch.Generator().manual_seed(4)).cuda() < 0.6
    finite, infinite = (x.masked_fill(gone, v) for v in (torch.finfo(torch.float32).min, -math.inf))
    for numbers in (dict(), dict(top_k=30), dict(top_p=0.9), dict(min_p=0.1)):
        for a, b in zip(slaq.sample_tokens(finite, u, **numbers), slaq.sample_tokens(infinite, u, **numbers)):
            assert a is None and b is None or torch.equal(a, b)
