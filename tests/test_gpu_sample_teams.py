"""Draws by each of the kernels that a call may be given to, in the sizes where one gives way to the next: registers of a warp up to 1,024 tokens; beyond, blocks of
128 threads for many short rows, of 256 for more rows than the GPU has SMs, of 512 for few.  Tolerances are those of test_gpu_sample_tokens."""

import pytest
import torch

from test_gpu_sample_tokens import FILTERS, TYPES, _check, _rows, slaq  # noqa: F401

pytestmark = pytest.mark.gpu

FLAT = [dict(top_k=1500), dict(top_p=0.97), dict(top_p=0.5), dict(min_p=1e-4), dict(top_k=2000, top_p=0.8), dict(top_k=3000, min_p=0.001), dict(top_p=0.999999),
        dict(top_k=3900, top_p=0.99, min_p=1e-5), dict(top_p=1.0)]


@pytest.mark.parametrize("numbers", [dict(), *FILTERS, dict(top_k=400, top_p=0.97), dict(top_p=0.9999)], ids=str)
@pytest.mark.parametrize("vocab", [65, 129, 257, 513, 700, 1023, 1024, 1025])
@pytest.mark.parametrize("dtype", TYPES)
def test_up_to_1024_tokens_and_one_more(slaq, dtype, vocab, numbers):  # noqa: F811
    for height, T in ((16.0, 0.8), (1.0, 4.0)):
        x, u = _rows(20, vocab, dtype, vocab, height=height, pad=vocab % 5, first=vocab % 3)
        _check(slaq.sample_tokens(x, u, T, **numbers), x, u, T, **numbers)


@pytest.mark.parametrize("numbers", FILTERS + [dict()], ids=str)
@pytest.mark.parametrize("vocab", [1025, 4000, 8180])
@pytest.mark.parametrize("dtype", TYPES)
def test_many_short_rows(slaq, dtype, vocab, numbers):  # noqa: F811
    x, u = _rows(300, vocab, dtype, vocab, height=16.0, pad=vocab % 7, first=vocab % 3)
    _check(slaq.sample_tokens(x, u, 0.8, **numbers), x, u, 0.8, **numbers)


@pytest.mark.parametrize("numbers", FLAT, ids=str)
@pytest.mark.parametrize("dtype", TYPES)
def test_many_short_rows_that_keep_much(slaq, dtype, numbers):  # noqa: F811
    for vocab, T in ((1025, 3.0), (4000, 1.0), (8180, 3.0)):
        x, u = _rows(300, vocab, dtype, 17, height=2.0, width=1.0)
        _check(slaq.sample_tokens(x, u, T, **numbers), x, u, T, **numbers)


@pytest.mark.parametrize("rows", [100, 149, 296, 297])
def test_the_same_rows_in_teams_of_every_size(slaq, rows):  # noqa: F811
    x, u = _rows(rows, 6000, torch.bfloat16, 5, height=10.0)
    for numbers in (dict(top_k=40, top_p=0.9), dict(top_p=0.9), dict(min_p=0.001), dict()):
        _check(slaq.sample_tokens(x, u, **numbers), x, u, **numbers)


@pytest.mark.parametrize("vocab", [1025, 3000, 8000])
@pytest.mark.parametrize("numbers", [dict(), dict(top_k=3), dict(top_p=0.37), dict(top_k=1100, top_p=0.61), dict(min_p=1.0), dict(top_p=0.9999), dict(top_p=0.0)], ids=str)
def test_equal_logits_in_many_short_rows(slaq, vocab, numbers):  # noqa: F811
    g = torch.Generator().manual_seed(vocab)
    u = torch.rand(300, generator=g).cuda()
    x = torch.full((300, vocab), -3.25, device="cuda", dtype=torch.bfloat16)
    x[100:, ::3] = -4.25
    x[200:, 1::3] = -3.75
    _check(slaq.sample_tokens(x, u, 0.7, **numbers), x, u, 0.7, **numbers)


def test_numbers_of_their_own_in_many_short_rows(slaq):  # noqa: F811
    rows, g = 400, torch.Generator().manual_seed(6)
    x, u = _rows(rows, 5000, torch.float32, 5, height=18.0)
    pick = lambda values, dtype: torch.tensor(values, dtype=dtype)[torch.randint(len(values), (rows,), generator=g)].cuda()   # noqa: E731
    numbers = dict(temperature=pick([0.0, 0.5, 1.0, 4.0], torch.float32), top_k=pick([-1, 0, 1, 7, 60, 2500], torch.int32), top_p=pick([0.0, 0.3, 0.9, 0.99, 1.0], torch.float32),
                   min_p=pick([0.0, 0.01, 0.2, 1.0], torch.float32))
    u[::9] = -1.0
    x[4] = float("-inf")
    x[5, 77] = float("nan")
    x[6, 77] = float("inf")
    _check(slaq.sample_tokens(x, u, **numbers), x, u, **numbers)
