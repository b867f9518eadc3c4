"""Rows of few tokens, of which a warp has several: every one has numbers of its own, and what one row is (greedy, not asked for, broken, behind the last) is
nothing to its neighbour."""

import math

import pytest
import torch

from test_gpu_sample_tokens import _check, _rows, slaq  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [1, 2, 3, 7, 10, 15, 16, 17, 31, 32, 33, 64, 100])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_neighbours_of_other_kinds(slaq, dtype, vocab):  # noqa: F811
    rows, g = 301, torch.Generator().manual_seed(vocab)
    x, u = _rows(rows, vocab, dtype, vocab, height=6.0)
    pick = lambda values, dtype: torch.tensor(values, dtype=dtype)[torch.randint(len(values), (rows,), generator=g)].cuda()   # noqa: E731
    numbers = dict(temperature=pick([0.0, 0.0, 0.7, 1.0, 2.0, math.nan], torch.float32), top_k=pick([0, 1, 3, 7], torch.int32),
                   top_p=pick([0.0, 0.5, 0.9, 1.0, 2.0], torch.float32), min_p=pick([0.0, 0.1, 1.0], torch.float32))
    u[::5] = -1.0
    x[3] = -math.inf
    x[8, vocab // 2] = math.nan
    x[12, 0] = math.inf
    _check(slaq.sample_tokens(x, u, **numbers), x, u, **numbers)
    only = dict(temperature=numbers["temperature"])
    _check(slaq.sample_tokens(x, u, **only), x, u, **only)
