"""min_p compares weights as 64 bits hold them: at temperatures far above the logits' differences all of them are 1, and so reach a min_p of 1, whatever kernel has the
row.  Tolerances are those of test_gpu_sample_tokens."""

import pytest
import torch

from test_gpu_sample_tokens import _check, _rows, slaq  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,vocab", [(12, 10), (12, 700), (12, 1500), (12, 5000), (12, 50_001), (305, 1500), (305, 4000), (305, 20_000)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_weights_that_round_to_1(slaq, dtype, rows, vocab):  # noqa: F811
    """.. with a few tokens that are masked, and a few whose weight is 0.5."""
    for T, size in ((1e30, 1.0), (1e20, 0.01), (0.1, 1e-24)):
        x, u = _rows(rows, vocab, dtype, vocab)
        x *= size
        x[:, ::7] = float("-inf")
        x[:, 1::5] = -0.6931471805599453 * T
        for numbers in (dict(min_p=1.0), dict(min_p=1.0, top_k=30), dict(min_p=1.0, top_k=1200), dict(min_p=0.9, top_p=0.9), dict(min_p=1.0, top_p=0.9), dict(min_p=1.0, top_k=2500, top_p=0.7),
                        dict(min_p=0.25)):
            _check(slaq.sample_tokens(x, u, T, **numbers), x, u, T, **numbers)


@pytest.mark.parametrize("rows", [12, 305])
@pytest.mark.parametrize("vocab", [700, 5000, 40_000])
def test_borders_of_min_p_between_neighbouring_logits(slaq, rows, vocab):  # noqa: F811
    """Logits are multiples of 1/64, so weights near a border lie 1.6 % apart, and rows keep from one token to nearly all."""
    x, u = _rows(rows, vocab, torch.float32, vocab, height=3.0, width=0.7)
    x.copy_(torch.round(x * 64) / 64)
    for q in (0.99, 0.7, 0.1, 1e-3, 1e-5, 1e-40):
        for numbers in (dict(min_p=q), dict(min_p=q, top_k=3 * vocab // 4)):
            _check(slaq.sample_tokens(x, u, **numbers), x, u, **numbers)
