"""Rows whose logits and temperature are far apart: neighbouring floating point numbers whose weights lie at the end of what 64 bits hold, and rows next to the
size from which on everything is decided in 64 bits.  Tolerances are those of test_gpu_sample_tokens."""

import math

import numpy as np
import pytest
import torch

from test_gpu_sample_tokens import _check, slaq  # noqa: F401

pytestmark = pytest.mark.gpu

NUMBERS = [dict(), dict(top_p=0.9), dict(top_k=7), dict(min_p=0.3), dict(top_k=25, top_p=0.6)]


def _steps_below(largest, rows, vocab, seed):
    """Every token is 0 to 30 floating point numbers below `largest`, a few are at it."""
    g = np.random.default_rng(seed)
    values = [np.float32(largest)]
    for _ in range(30):
        values.append(np.nextafter(values[-1], np.float32(-np.inf)))
    values = np.array(values)
    assert np.isfinite(values).all()
    x = values[g.integers(1, 31, (rows, vocab))]
    x[np.arange(rows), g.integers(0, vocab, rows)] = values[0]
    return torch.from_numpy(x).cuda(), torch.from_numpy(g.random(rows, dtype=np.float32)).cuda()


@pytest.mark.parametrize("vocab", [10, 33, 700, 1024, 5000])
@pytest.mark.parametrize("largest", [20.0, 1.0, 1.5, -3.0, 1e-20, 6e4, 1e30, -1e30])
def test_weights_at_the_end_of_64_bits(slaq, vocab, largest):  # noqa: F811
    """693 temperatures, where weights come to their end, are half a step between neighbouring numbers, a few, many."""
    step = float(np.float32(largest) - np.nextafter(np.float32(largest), np.float32(-np.inf)))
    x, u = _steps_below(largest, 12, vocab, vocab)
    for steps in (0.5, 0.9, 1.0, 1.1, 1.9, 2.5, 3.7, 8.0, 15.3, 30.0):
        T = step / 693.0 * steps
        if not 1e-30 <= T <= 1e30:
            continue
        for numbers in NUMBERS:
            _check(slaq.sample_tokens(x, u, T, **numbers), x, u, T, **numbers)


@pytest.mark.parametrize("vocab", [10, 33, 70, 700, 1023, 5000])
@pytest.mark.parametrize("T", [1.4e28, 1.6e28, 2e29, 1e30])
def test_the_lowest_logits_at_the_highest_temperatures(slaq, vocab, T):  # noqa: F811
    g = np.random.default_rng(vocab)
    low = np.finfo(np.float32).min
    x = (low * (1 - g.random((12, vocab)) * 20.0 * T / 3.4e38)).astype(np.float32)
    x[3:6, ::2] = low
    x[6:9, 1::3] = -math.inf
    x, u = torch.from_numpy(x).cuda(), torch.from_numpy(g.random(12, dtype=np.float32)).cuda()
    for numbers in NUMBERS:
        _check(slaq.sample_tokens(x, u, T, **numbers), x, u, T, **numbers)


@pytest.mark.parametrize("vocab", [1500, 20_000])
@pytest.mark.parametrize("off", [-40.0, -3.0, 0.0, 3.0, 40.0])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_where_32_bits_give_way(slaq, vocab, off, sign):  # noqa: F811
    """The largest logit is 2^22 octaves of the weight from 0, a little less, a little more; logits there are multiples of 1/4."""
    border = sign * (2.0 ** 22 * math.log(2.0) + off)
    g = torch.Generator().manual_seed(vocab)
    x = torch.randn(12, vocab, generator=g) * 2
    x[torch.arange(12), torch.randint(vocab, (12,), generator=g)] += 16.0 * torch.rand(12, generator=g)
    x = torch.round((x.double() - x.double().amax(1, keepdim=True) + border) * 4).div(4).float().cuda()
    u = torch.rand(12, generator=g).cuda()
    for numbers in [*NUMBERS, dict(top_p=0.99)]:
        _check(slaq.sample_tokens(x, u, **numbers), x, u, **numbers)
