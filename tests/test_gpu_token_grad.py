"""The gradient of log probabilities and entropies, alone and in one pass with the loss, against 64 bits and differences.

Tolerances (u = 2^-24).  p = exp(scale (x - m)) / S: argument 3u|d|, exponential 4u, S (44 + V/256) u, division and product 2u:
p is within (50 + V/256 + 3|d|) u p, and p|d| <= 0.37 + p ln V.  The rest is a handful of products, all relative to |g| (1 + p)
or |h| p (|ln p| + H) <= |h| (0.37 + 2 ln V).  Behind it one rounding to the type: eps/2 of the value (fp16 below 2^-14: 2^-25)."""

import math

import pytest
import torch

import token_rows as ref
from test_gpu_token_logprobs import TYPES, U, _rows, slaq  # noqa: F401

pytestmark = pytest.mark.gpu


def _check(got, want, vocab, g, h, scale):
    got = got.double().cpu()
    rows_g = g.double().abs().cpu()[:, None]
    rows_h = torch.zeros_like(rows_g) if h is None else h.double().abs().cpu()[:, None]
    ln = math.log(vocab) + 1
    tol = (rows_g * (60 + vocab / 256 + 4 * ln) + rows_h * (70 + vocab / 256 + 4 * ln) * (1 + 2 * ln)) * U * scale
    return got, want, tol


def _near(got, want, tol, dtype):
    tol = tol + torch.finfo(dtype).eps / 2 * want.abs() + (2.0 ** -25 if dtype == torch.float16 else 0.0)
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    off = (got - want).abs()
    ok = bool((same | (off <= tol)).all())
    assert ok, float((off - tol)[~same].max())


def _grads(rows, gen):
    return torch.randn(rows, generator=gen).cuda(), torch.randn(rows, generator=gen).cuda()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [1, 2, 9, 10, 33, 100, 256, 1000, 1025, 2047, 4100, 32768, 50001])
def test_gradients_of_every_length(slaq, vocab, dtype):  # noqa: F811
    for rows, pad, scale in ((1, 0, 1.0), (5, 1, 0.7), (19, 8, 1.3)):
        x, t, gen = _rows(rows, vocab, dtype, pad, vocab + rows)
        g, h = _grads(rows, gen)
        parts = slaq.token_logprobs(x, t, scale=scale)
        for with_entropy in (False, True):
            kw = dict(entropy=parts.entropy, grad_entropy=h) if with_entropy else {}
            got = slaq.token_logprobs_grad(x, t, parts.norm, g, scale=scale, **kw)
            _near(*_check(got, ref.gradient(x, t, g, h if with_entropy else None, scale), vocab, g, h if with_entropy else None, scale), dtype)
        logprob, got = slaq.token_loss(x, t, g, scale=scale)
        _near(*_check(got, ref.gradient(x, t, g, None, scale), vocab, g, None, scale), dtype)
        torch.testing.assert_close(logprob, parts.logprob, rtol=4 * U, atol=2 * (40 + vocab / 256) * U)


@pytest.mark.parametrize("vocab,dtype", [(130001, torch.bfloat16), (262144, torch.float32), (1 << 20, torch.bfloat16), (700001, torch.float32)])
def test_long_rows(slaq, vocab, dtype):  # noqa: F811
    x, t, gen = _rows(2, vocab, dtype, 3, vocab)
    g, h = _grads(2, gen)
    parts = slaq.token_logprobs(x, t)
    got = slaq.token_logprobs_grad(x, t, parts.norm, g, entropy=parts.entropy, grad_entropy=h)
    _near(*_check(got, ref.gradient(x, t, g, h), vocab, g, h, 1.0), dtype)
    logprob, got = slaq.token_loss(x, t, g)
    _near(*_check(got, ref.gradient(x, t, g), vocab, g, None, 1.0), dtype)
    torch.testing.assert_close(logprob, parts.logprob, rtol=4 * U, atol=2 * (40 + vocab / 256) * U)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [5, 40, 300, 3000, 40000])
def test_masked_rows(slaq, vocab, dtype):  # noqa: F811
    x, t, gen = _rows(14, vocab, dtype, 3, vocab)
    g, h = _grads(14, gen)
    low, k = torch.finfo(dtype).min, vocab // 2
    x[1, k:] = -math.inf
    x[2, :k] = low
    x[3] = -math.inf
    x[4] = low
    x[5, k] = math.nan
    x[6, k] = math.inf
    x[7] = -math.inf
    x[7, vocab - 1] = 2.0
    x[8, 0] = -math.inf
    t[8], t[7] = 0, vocab - 1
    t[9], t[10], t[11], t[12] = -1, -7, vocab, vocab - 1
    x[10] = math.nan
    t[13] = 0
    x[13] = -math.inf
    x[13, 0] = low
    parts = slaq.token_logprobs(x, t)
    want = ref.gradient(x, t, g, h)
    got = slaq.token_logprobs_grad(x, t, parts.norm, g, entropy=parts.entropy, grad_entropy=h)
    _near(*_check(got, want, vocab, g, h, 1.0), dtype)
    logprob, got = slaq.token_loss(x, t, g)
    _near(*_check(got, ref.gradient(x, t, g), vocab, g, None, 1.0), dtype)
    same = (logprob == parts.logprob) | (logprob.isnan() & parts.logprob.isnan())
    assert bool((same | ((logprob - parts.logprob).abs() <= 4 * U * parts.logprob.abs() + 2 * (40 + vocab / 256) * U)).all())


@pytest.mark.parametrize("vocab", [10, 600, 8000, 120000])
def test_a_factor_of_zero_leaves_zeros(slaq, vocab):  # noqa: F811
    x, t, _ = _rows(3, vocab, torch.bfloat16, 0, 1)
    zero = torch.zeros(3, device="cuda")
    parts = slaq.token_logprobs(x, t)
    assert not slaq.token_loss(x, t, zero)[1].any()
    assert not slaq.token_logprobs_grad(x, t, parts.norm, zero, entropy=parts.entropy, grad_entropy=zero).any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,pad", [(10, 0), (777, 0), (777, 3), (8192, 0), (50001, 0), (50001, 7), (200000, 8), (900001, 0)])
def test_in_the_place_of_the_logits(slaq, vocab, pad, dtype):  # noqa: F811
    x, t, gen = _rows(6, vocab, dtype, pad, 2)
    g, h = _grads(6, gen)
    t[2] = -1
    parts = slaq.token_logprobs(x, t)
    want = slaq.token_loss(x, t, g)
    y = x.clone() if pad == 0 else torch.empty(6, vocab + pad, dtype=dtype, device="cuda").copy_(torch.nn.functional.pad(x, (0, pad), value=7.0))[:, :vocab]
    got = slaq.token_loss(y, t, g, out=y)
    assert got[1].data_ptr() == y.data_ptr()
    assert torch.equal(got[0], want[0]) and torch.equal(y, want[1])
    if pad:
        assert bool((y.as_strided((6, pad), (vocab + pad, 1), vocab) == 7.0).all())       # what lies behind a row stays
    y = x.clone()
    want = slaq.token_logprobs_grad(x, t, parts.norm, g, entropy=parts.entropy, grad_entropy=h)
    slaq.token_logprobs_grad(y, t, parts.norm, g, entropy=parts.entropy, grad_entropy=h, out=y)
    assert torch.equal(y, want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [65, 66, 125, 126, 171, 249, 250, 253, 254, 505, 506, 509, 510, 1017, 1018, 1025, 2500, 9001, 70003])
def test_alignments_that_differ(slaq, vocab, dtype):  # noqa: F811
    """Logits and gradient each at its own distance from 16 bytes: every pair of distances gives the bits of any other."""
    step = 16 // dtype.itemsize
    x, t, gen = _rows(7, vocab, dtype, 0, vocab)
    g, h = _grads(7, gen)
    t[3], t[4], t[5], t[6] = -1, 0, vocab - 1, vocab
    x[2, vocab // 3:] = -math.inf
    pitch = (vocab + 3 * step) // step * step
    places = torch.full((2, 7, pitch), 5.0, dtype=dtype, device="cuda")
    where = range(0, step) if vocab < 3000 else (0, 1, step - 1)
    expected = {}
    for at in where:
        y = places[0, :, at:at + vocab].copy_(x)
        parts = slaq.token_logprobs(y, t)
        for to in where:
            for name in ("loss", "grad", "entropy"):
                places[1] = 5.0
                out = places[1, :, to:to + vocab]
                if name == "loss":
                    slaq.token_loss(y, t, g, out=out)
                else:
                    kw = dict(entropy=parts.entropy, grad_entropy=h) if name == "entropy" else {}
                    slaq.token_logprobs_grad(y, t, parts.norm, g, out=out, **kw)
                assert bool((places[1, :, :to] == 5.0).all()) and bool((places[1, :, to + vocab:] == 5.0).all())
                want = expected.setdefault((name, at), out.clone())       # the sums' order is the logits', not the gradient's
                assert torch.equal(torch.nan_to_num(out), torch.nan_to_num(want)) and bool((out[6] != out[6]).all())
                if to == at:
                    rows = slice(0, 6)
                    with_h = h[rows] if name == "entropy" else None
                    _near(*_check(out[rows], ref.gradient(y[rows], t[rows], g[rows], with_h), vocab, g[rows], with_h, 1.0), dtype)


def test_rows_that_alternate_with_the_logits(slaq):  # noqa: F811
    both = torch.randn(5, 2 * 3000, generator=torch.Generator().manual_seed(1)).cuda()
    x, out = both[:, :3000], both[:, 3000:]
    t, g = torch.arange(5, device="cuda"), torch.randn(5, generator=torch.Generator().manual_seed(2)).cuda()
    before = x.clone()
    want = slaq.token_loss(before, t, g)[1]
    assert torch.equal(slaq.token_loss(x, t, g, out=out)[1], want) and torch.equal(x, before)


def test_differences(slaq):  # noqa: F811
    """Central differences in 64 bits of the definition, of step 1e-5: their own error is about 1e-10 of the largest third
    derivative (below 1); the gradient's is its 1e-5."""
    x, t, gen = _rows(3, 12, torch.float32, 0, 8, std=1.0)
    g, h = _grads(3, gen)
    parts = slaq.token_logprobs(x, t, scale=1.4)
    got = slaq.token_logprobs_grad(x, t, parts.norm, g, entropy=parts.entropy, grad_entropy=h, scale=1.4).double().cpu()

    def value(y):
        r = ref.logprobs(y, t, 1.4)
        return r["logprob"] * g.double().cpu() + r["entropy"] * h.double().cpu()
    for i in range(12):
        step = torch.zeros(3, 12, dtype=torch.float64)
        step[:, i] = 1e-5
        slope = (value(x.double().cpu() + step) - value(x.double().cpu() - step)) / 2e-5
        torch.testing.assert_close(got[:, i], slope, rtol=1e-5, atol=1e-5)


def test_in_a_graph_and_on_a_stream(slaq):  # noqa: F811
    x, t, gen = _rows(33, 7001, torch.bfloat16, 0, 4)
    g, _ = _grads(33, gen)
    want = slaq.token_loss(x, t, g)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = slaq.token_loss(x, t, g, stream=side)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    graph, y = torch.cuda.CUDAGraph(), x.clone()
    with torch.cuda.graph(graph):
        parts = slaq.token_logprobs(y, t)
        got = slaq.token_logprobs_grad(y, t, parts.norm, g)
        slaq.token_loss(y, t, g, out=y)
    for _ in range(2):
        y.copy_(x)
        graph.replay()
        assert torch.equal(y, want[1])
        _near(got.double().cpu(), want[1].double().cpu(), torch.tensor(1e-4), torch.bfloat16)


def test_refusals(slaq):  # noqa: F811
    x, t, gen = _rows(6, 100, torch.float32, 0, 1)
    g, h = _grads(6, gen)
    parts = slaq.token_logprobs(x, t)
    flat = torch.zeros(2000, device="cuda")
    a, b = flat[:600].view(6, 100), flat[50:650].view(6, 100)
    for call in (lambda: slaq.token_loss(a, t, g, out=b), lambda: slaq.token_loss(x, t, None), lambda: slaq.token_loss(x, None, g),
                 lambda: slaq.token_loss(x, t, g, out=x.half()), lambda: slaq.token_loss(x, t, g, out=flat[:100].expand(6, 100)),
                 lambda: slaq.token_loss(flat[:100].expand(6, 100), t, g, out=flat[:600].view(6, 100)),
                 lambda: slaq.token_logprobs_grad(x, t, parts.norm, g, grad_entropy=h), lambda: slaq.token_logprobs_grad(x, t, None, g),
                 lambda: slaq.token_logprobs_grad(x, t, parts.norm, g.double()), lambda: slaq.token_loss(x, t, g, scale=-1.0)):
        with pytest.raises(slaq.SlaqError) as e:
            call()
        assert e.value.code == -1
