"""Drawn tokens against the definition in 64 bits, row by row.

A token, and how many are kept, are whole numbers and have to be equal.  The definition itself decides by sums of up to 2^22 rounded terms (2^-53 each and
2^-53 for every addition): rows in which a decision lies within 2^-40 of a border are left out, which no row below is.
Log probabilities (u = 2^-24): the sum's bound is 5u of additions, 4u of the exponential and 1.4u |t| of the exponents, log2 of the
vocabulary at the most: (9 + 1.4 * 22) u = 40u of the sum, hence 40u of its logarithm, and one rounding."""

import math

import numpy as np
import pytest
import torch

import sampling

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def slaq():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_1802_04819_b200 as mod
    mod.build()
    return mod


def _rows(rows, vocab, dtype, seed, height=8.0, width=2.0, pad=0, first=0):
    """Rows of every height of their likely tokens; `pad` columns behind them, the first element at `first` of the buffer."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, vocab, generator=g) * width
    x[torch.arange(rows), torch.randint(vocab, (rows,), generator=g)] += height * torch.rand(rows, generator=g)
    buffer = torch.zeros(first + rows * (vocab + pad), dtype=dtype)
    out = buffer[first:].view(rows, vocab + pad)[:, :vocab]
    out.copy_(x.to(dtype))
    on = buffer.cuda()
    return on[first:].view(rows, vocab + pad)[:, :vocab], torch.rand(rows, generator=g).cuda()


def _each(value, none, row):
    if value is None:
        return none
    return float(value[row]) if torch.is_tensor(value) else value


def _check(got, x, uniform, temperature=1.0, top_k=None, top_p=None, min_p=None):
    x, u = x.double().cpu().numpy(), uniform.cpu().numpy()
    columns = [temperature, top_k, top_p, min_p]
    columns = [c.cpu() if torch.is_tensor(c) else c for c in columns]
    token, logprob, kept_logprob = (t.cpu().numpy() for t in got[:3])
    kept = None if got.kept is None else got.kept.cpu().numpy()
    for r in range(x.shape[0]):
        T, k, p, q = (_each(c, none, r) for c, none in zip(columns, (1.0, 0, 1.0, 0.0)))
        want = sampling.draw(x[r], u[r], T, int(k), p, q)
        assert want[4] > 2.0 ** -40, (r, want)
        assert token[r] == want[0], (r, token[r], want, T, k, p, q)
        if kept is not None:
            assert kept[r] == want[3], (r, kept[r], want, T, k, p, q)
        for mine, exact in ((logprob[r], want[1]), (kept_logprob[r], want[2])):
            if math.isfinite(exact):
                assert abs(mine - exact) <= 40 * U + U * abs(exact), (r, mine, exact)
            else:
                np.testing.assert_equal(mine, np.float32(exact))


FILTERS = [dict(top_k=1), dict(top_k=50), dict(top_p=0.9), dict(min_p=0.05), dict(top_k=20, top_p=0.7, min_p=0.1), dict(top_p=0.0), dict(top_k=10 ** 6, top_p=1.0, min_p=0.0)]
VOCABS = [1, 2, 3, 10, 31, 33, 64, 100, 171, 500, 2047, 2048, 2049, 5000, 50_001]


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("dtype", TYPES)
def test_the_whole_distribution(slaq, dtype, vocab):
    rows = 300 if vocab < 3000 else 60
    for T, pad, first in ((1.0, 0, 0), (0.6, 3, 1), (torch.full((rows,), 1.5, device="cuda"), 8, 5)):
        x, u = _rows(rows, vocab, dtype, vocab + first, pad=pad, first=first)
        got = slaq.sample_tokens(x, u, T)
        assert got.kept is None
        _check(got, x, u, T)


@pytest.mark.parametrize("numbers", FILTERS, ids=str)
@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("dtype", TYPES)
def test_what_is_kept(slaq, dtype, vocab, numbers):
    x, u = _rows(40, vocab, dtype, vocab, height=16.0, pad=vocab % 5, first=vocab % 3)
    _check(slaq.sample_tokens(x, u, 0.8, **numbers), x, u, 0.8, **numbers)


@pytest.mark.parametrize("numbers", [dict(top_k=5000), dict(top_p=0.97), dict(top_p=0.5), dict(min_p=1e-4), dict(top_k=6000, top_p=0.8), dict(top_k=9000, min_p=0.001),
                                     dict(top_p=0.999999), dict(top_k=40_000, top_p=0.99, min_p=1e-5), dict(top_k=19_999), dict()], ids=str)
@pytest.mark.parametrize("dtype", TYPES)
def test_more_is_kept_than_a_list_holds(slaq, dtype, numbers):
    """Flat rows of 20,000 and 130,001 tokens; bf16 has hundreds of equal logits at every border."""
    for rows, vocab, T in ((12, 20_000, 1.0), (6, 130_001, 3.0)):
        x, u = _rows(rows, vocab, dtype, 17, height=2.0, width=1.0)
        _check(slaq.sample_tokens(x, u, T, **numbers), x, u, T, **numbers)


@pytest.mark.parametrize("vocab", [7, 100, 3000, 20_000])
@pytest.mark.parametrize("numbers", [dict(), dict(top_k=3), dict(top_p=0.37), dict(top_k=2500, top_p=0.61), dict(min_p=1.0), dict(top_p=0.9999)], ids=str)
def test_equal_logits_go_by_their_ids(slaq, vocab, numbers):
    """All equal, and two values: the weights of the larger are 1, so 1/3 of them decides where sums in 32 bits would do."""
    g = torch.Generator().manual_seed(vocab)
    u = torch.rand(40, generator=g).cuda()
    for value in (0.0, -3.25, 11.0):
        x = torch.full((40, vocab), value, device="cuda", dtype=torch.bfloat16)
        _check(slaq.sample_tokens(x, u, 0.7, **numbers), x, u, 0.7, **numbers)
        x[:, ::3] = value - 1.0
        x[:, 1::3] = torch.where(torch.rand(40, 1, generator=g) < 0.5, value, value - 0.5).to(x)
        _check(slaq.sample_tokens(x, u, 0.7, **numbers), x, u, 0.7, **numbers)


def test_a_zero_of_either_sign_is_the_same(slaq):
    x = torch.zeros(8, 5000, device="cuda")
    x[:, ::2] = -0.0
    u = torch.linspace(0.01, 0.98, 8, device="cuda")
    for numbers in (dict(top_k=4), dict(top_p=0.31), dict(top_k=2999), dict()):
        _check(slaq.sample_tokens(x, u, **numbers), x, u, **numbers)


@pytest.mark.parametrize("vocab", [40, 3000, 30_000])
def test_rows_with_numbers_of_their_own(slaq, vocab):
    rows, g = 200, torch.Generator().manual_seed(vocab)
    x, u = _rows(rows, vocab, torch.float32, 5, height=18.0)
    pick = lambda values, dtype: torch.tensor(values, dtype=dtype)[torch.randint(len(values), (rows,), generator=g)].cuda()   # noqa: E731
    numbers = dict(temperature=pick([0.0, 0.5, 1.0, 2.0], torch.float32), top_k=pick([-1, 0, 1, 7, 60, 2500], torch.int32), top_p=pick([0.0, 0.3, 0.9, 0.99, 1.0], torch.float32),
                   min_p=pick([0.0, 0.01, 0.2, 1.0], torch.float32))
    u[::9] = -1.0
    _check(slaq.sample_tokens(x, u, **numbers), x, u, **numbers)
    only = {k: v for k, v in numbers.items() if k == "temperature"}
    _check(slaq.sample_tokens(x, u, **only), x, u, **only)


def test_numbers_out_of_range_are_their_rows_matter(slaq):
    bad = [dict(temperature=-1.0), dict(temperature=math.nan), dict(temperature=1e-31), dict(temperature=1e31), dict(temperature=math.inf), dict(top_p=-0.1), dict(top_p=1.1),
           dict(top_p=math.nan), dict(min_p=-0.1), dict(min_p=1.5), dict(min_p=math.nan), dict(uniform=1.0), dict(uniform=math.nan), dict(uniform=math.inf), dict(uniform=-0.5), dict()]
    for vocab in (20, 3000):
        x, u = _rows(len(bad), vocab, torch.float32, 1)
        columns = dict(temperature=torch.full((len(bad),), 0.9), top_p=torch.full((len(bad),), 0.9), min_p=torch.full((len(bad),), 0.01), uniform=u.cpu())
        for r, change in enumerate(bad):
            for name, value in change.items():
                columns[name][r] = value
        columns = {k: v.cuda() for k, v in columns.items()}
        u = columns.pop("uniform")
        got = slaq.sample_tokens(x, u, **columns)
        _check(got, x, u, **columns)
        assert got.token[:-2].eq(-1).all() and got.token[-1] >= 0 and got.logprob[-2] == 0
        got = slaq.sample_tokens(x, u, columns["temperature"])
        _check(got, x, u, columns["temperature"])


def test_masked_and_broken_rows(slaq):
    for vocab in (1, 5, 40, 3000, 20_000):
        x, u = _rows(10, vocab, torch.float16, vocab)
        x[0] = -math.inf
        x[1, vocab // 2] = math.nan
        x[2, vocab // 2] = math.inf
        x[3, : vocab - 1] = -math.inf
        x[4, vocab // 2:] = -math.inf
        x[5, : vocab // 2] = -math.inf
        x[6] = torch.finfo(torch.float16).min
        x[7, ::2] = torch.finfo(torch.float16).min
        for numbers in (dict(), dict(top_k=4, top_p=0.9), dict(top_k=vocab - 1), dict(min_p=0.1), dict(top_p=0.8), dict(temperature=0.0)):
            _check(slaq.sample_tokens(x, u, **numbers), x, u, **numbers)


@pytest.mark.parametrize("T", [1e-30, 1e-6, 0.01, 100.0, 1e30])
@pytest.mark.parametrize("size", [1e-30, 1.0, 1e4, 1e30])
def test_logits_and_temperatures_of_any_size(slaq, T, size):
    """Beyond |x / T| = 2^16 or so everything is decided in 64 bits."""
    for vocab in (33, 5000):
        x, u = _rows(20, vocab, torch.float32, 3)
        x *= size
        for numbers in (dict(), dict(top_p=0.6), dict(top_k=7, min_p=0.3)):
            _check(slaq.sample_tokens(x, u, T, **numbers), x, u, T, **numbers)


def test_uniforms_at_the_ends(slaq):
    x, _ = _rows(4, 6000, torch.float32, 2)
    u = torch.tensor([0.0, 2.0 ** -149, 2.0 ** -24, 1.0 - 2.0 ** -24], device="cuda")
    x[:, 0] = -60.0        # its weight in 64 bits is not 0
    for numbers in (dict(), dict(top_p=0.99), dict(top_k=10)):
        got = slaq.sample_tokens(x, u, **numbers)
        for r in range(4):
            want = sampling.draw(x[r].double().cpu().numpy(), float(u[r]), 1.0, numbers.get("top_k", 0), numbers.get("top_p", 1.0))
            assert int(got.token[r]) == want[0]


def test_tokens_next_to_a_border_are_decided_in_64_bits(slaq):
    """Random numbers on the border between two tokens, as near as 32 bits come: an error of 2^-22 in a sum would take the wrong one in most rows."""
    g = torch.Generator().manual_seed(8)
    for vocab in (300, 9000):
        x = (torch.randn(1, vocab, generator=g) * 0.5).expand(64, vocab).contiguous()
        w = np.exp(x[0].double().numpy() - float(x[0].max()))
        run = np.cumsum(w) / w.sum()
        at = torch.randint(vocab // 3, vocab, (64,), generator=g).numpy()
        u = torch.from_numpy(np.nextafter(run[at].astype(np.float32), np.where(np.arange(64) % 2, 0, 1).astype(np.float32)))
        got = slaq.sample_tokens(x.cuda(), u.cuda())
        want = [sampling.draw(x[r].double().numpy(), float(u[r]))[0] for r in range(64)]
        assert got.token.tolist() == want
        got = slaq.sample_tokens(x.cuda(), u.cuda(), top_p=1.0)
        assert got.token.tolist() == want


def test_shares_next_to_a_border(slaq):
    g = torch.Generator().manual_seed(9)
    for vocab in (300, 9000):
        x = (torch.randn(1, vocab, generator=g) * 3).expand(64, vocab).contiguous()
        w = np.sort(np.exp(x[0].double().numpy() - float(x[0].max())))[::-1]
        run = np.cumsum(w) / w.sum()
        at = np.arange(64) * vocab // 100
        p = torch.from_numpy(np.nextafter(run[at].astype(np.float32), np.where(np.arange(64) % 2, 0, 1).astype(np.float32)))
        u = torch.rand(64, generator=g)
        got = slaq.sample_tokens(x.cuda(), u.cuda(), top_p=p.cuda())
        assert got.kept.tolist() == [sampling.draw(x[r].double().numpy(), float(u[r]), p=float(p[r]))[3] for r in range(64)]


def test_strides_and_a_single_row(slaq):
    g = torch.Generator().manual_seed(3)
    x = torch.randn(3, 4000, generator=g).cuda().bfloat16()
    u = torch.rand(3, generator=g).cuda()
    same = x[1:2].expand(3, 4000)
    _check(slaq.sample_tokens(same, u, top_p=0.9), same, u, top_p=0.9)
    _check(slaq.sample_tokens(x[2:, 5:3333], u[:1]), x[2:, 5:3333], u[:1])
    column = x[:, 7:8]
    _check(slaq.sample_tokens(column, u), column, u)
    none = slaq.sample_tokens(x[:0], u[:0], top_k=3)
    assert none.token.shape == (0,) and none.kept.shape == (0,)


def test_the_draws_follow_the_distribution(slaq):
    """200,000 draws of 8 tokens: each token's share within 5 standard deviations of its probability."""
    x = torch.tensor([2.0, 1.0, 0.0, -1.0, 3.0, -2.0, 0.5, 1.5]).cuda()
    n = 200_000
    u = torch.rand(n, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    p = torch.softmax(x.double(), 0)
    share = torch.bincount(slaq.sample_tokens(x.expand(n, 8), u).token, minlength=8).double() / n
    assert bool(((share - p).abs() < 5 * (p * (1 - p) / n).sqrt()).all())


def test_log_probabilities_are_those_of_the_scoring_call(slaq):
    x, u = _rows(50, 10_000, torch.bfloat16, 4)
    got = slaq.sample_tokens(x, u, 0.5, top_k=40)
    scored = slaq.token_logprobs(x, got.token, scale=2.0)
    # each within 40u + u |lp| of the exact one
    assert bool(((got.logprob - scored.logprob).abs() <= 80 * U + 2 * U * scored.logprob.abs()).all())


def test_captured_and_on_other_streams(slaq):
    x, u = _rows(30, 5000, torch.bfloat16, 6)
    slaq.sample_tokens(x, u, 0.9, top_p=0.9)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got, plain = slaq.sample_tokens(x, u, 0.9, top_p=0.9), slaq.sample_tokens(x, u)
    for seed in (1, 2):
        y, v = _rows(30, 5000, torch.bfloat16, seed)
        x.copy_(y)
        u.copy_(v)
        graph.replay()
        _check(got, x, u, 0.9, top_p=0.9)
        _check(plain, x, u)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (side, side.cuda_stream):
        got = slaq.sample_tokens(x, u, stream=stream)
        side.synchronize()
        _check(got, x, u)


def test_refusals(slaq):
    x, u = _rows(4, 100, torch.float32, 1)
    f, i = torch.ones(4, device="cuda"), torch.ones(4, dtype=torch.int32, device="cuda")
    for bad in (lambda: slaq.sample_tokens(x, None), lambda: slaq.sample_tokens(x, u, None), lambda: slaq.sample_tokens(x, u[:3]), lambda: slaq.sample_tokens(x, u.double()),
                lambda: slaq.sample_tokens(x.double(), u), lambda: slaq.sample_tokens(x[0], u), lambda: slaq.sample_tokens(x.t(), u), lambda: slaq.sample_tokens(x.cpu(), u),
                lambda: slaq.sample_tokens(x[:, :0], u), lambda: slaq.sample_tokens(x, u, -1.0), lambda: slaq.sample_tokens(x, u, 1e31), lambda: slaq.sample_tokens(x, u, math.nan),
                lambda: slaq.sample_tokens(x, u, top_p=1.5), lambda: slaq.sample_tokens(x, u, top_p=-0.1), lambda: slaq.sample_tokens(x, u, min_p=2.0),
                lambda: slaq.sample_tokens(x, u, top_k=f), lambda: slaq.sample_tokens(x, u, top_p=i), lambda: slaq.sample_tokens(x, u, i), lambda: slaq.sample_tokens(x, u, top_k=i[:2])):
        with pytest.raises(slaq.SlaqError):
            bad()
