"""Shares of equal weights that come out whole in 64 bits: top_p times the sum is rounded, as the definition's product is, before anything is compared with it.
Weights are 1 or 0 and their sums whole numbers, so the definition's own decisions are exact however near to a border they lie."""

import math

import pytest
import torch

import sampling
from test_gpu_sample_tokens import U, slaq  # noqa: F401

pytestmark = pytest.mark.gpu


def _check_whole(got, x, u, top_p, top_k=0, T=1.0):
    for r in range(x.shape[0]):
        token, logprob, kept_logprob, kept, _ = sampling.draw(x[r].double().cpu().numpy(), float(u[r]), T, k=top_k, p=top_p)
        assert (int(got.token[r]), int(got.kept[r])) == (token, kept), (r, top_p, top_k)
        for mine, exact in ((float(got.logprob[r]), logprob), (float(got.kept_logprob[r]), kept_logprob)):
            assert math.isfinite(mine) and abs(mine - exact) <= 40 * U + U * abs(exact)      # as in test_gpu_sample_tokens


@pytest.mark.parametrize("rows,vocab", [(r, v) for r in (2, 160, 300) for v in (10, 20, 30, 50, 100, 130, 400, 1000, 1100, 2000, 5000, 6000, 20_000)] + [(2, 130_000)])
def test_whole_shares_of_equal_logits(slaq, rows, vocab):  # noqa: F811
    """Tenths, some of whose products with whole numbers lie beside the whole number that they round to.  Masked tokens in between, of either kind."""
    g = torch.Generator().manual_seed(vocab)
    u = torch.rand(rows, generator=g)
    asked = torch.zeros(rows, dtype=torch.bool)
    asked[:: max(1, rows // 8)] = True
    u = torch.where(asked, u, -1.0).cuda()
    for masked in (None, float("-inf"), torch.finfo(torch.float32).min):
        x = torch.full((rows, vocab), 1.25)
        if masked is not None:
            x[:, torch.randperm(vocab, generator=g)[: vocab // 5]] = masked
        x = x.cuda()
        for p in (0.1, 0.3, 0.55, 0.6, 0.7, 0.9, 0.95, 0.99):
            for numbers in (dict(top_p=p), dict(top_p=p, top_k=4 * vocab // 10)):
                _check_whole(slaq.sample_tokens(x, u, **numbers), x, u, **numbers)


@pytest.mark.parametrize("rows,vocab", [(r, v) for r in (2, 160, 300) for v in (10, 30, 50, 100, 400, 1000, 5000, 6000, 20_000)])
def test_whole_shares_of_logits_far_below_the_temperature(slaq, rows, vocab):  # noqa: F811
    """Four values, all of whose weights are 1: the border lies among the equal ones of one value, behind all of another."""
    g = torch.Generator().manual_seed(vocab)
    u = torch.full((rows,), -1.0)
    u[:: max(1, rows // 8)] = 0.37
    u = u.cuda()
    x = torch.tensor([-1.5, 0.0, 0.25, 3.0])[torch.randint(4, (rows, vocab), generator=g)]
    x[:, torch.randperm(vocab, generator=g)[: vocab // 5]] = torch.finfo(torch.float32).min
    x = x.cuda()
    for p in (0.1, 0.3, 0.55, 0.6, 0.7, 0.9, 0.95, 0.99):
        for numbers in (dict(top_p=p), dict(top_p=p, top_k=4 * vocab // 10)):
            _check_whole(slaq.sample_tokens(x, u, 1e30, **numbers), x, u, T=1e30, **numbers)
