"""Log probabilities, entropies and top alternatives against 64 bits.

Tolerances, by counting roundings (u = 2^-24).  Inputs are exact.  d = scale (x - m): two roundings, 2u|d|.  A term e = exp d:
its argument is off by at most 3u|d| (the constant's rounding too), the exponential itself by 2^-22 = 4u; since e|d| <= 0.37,
the sum S of V terms is off by (4 + 2 + n) u S where n counts the additions that a term passes through: at most V / 256 in
a thread and 32 behind that.  ln S: that, and half an ulp.  So a log probability is within
2u|d| + (40 + V/256) u + u |value|, and the entropy (terms e|d|, summed alike, two divisions and products, value <= ln V) within
(48 + V/256) u (1 + value)."""

import math

import pytest
import torch

import token_rows as ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def slaq():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_1802_04819_b200 as mod
    mod.build()
    return mod


def _rows(rows, vocab, dtype, pad, seed, std=3.0):
    g = torch.Generator().manual_seed(seed)
    wide = (torch.randn(rows, vocab + pad, generator=g) * std).to(dtype)
    return wide.cuda()[:, :vocab], torch.randint(vocab, (rows,), generator=g).cuda(), g


def _check(got, want, vocab, x, scale, top):
    n = (40 + vocab / 256) * U
    m = want["norm"][:, :1]
    far = torch.where(torch.isfinite(m), ((x.double().cpu().clamp_min(-1e30) - m) * scale).abs(), torch.zeros_like(m))

    def near(a, b, tol, what):
        a = a.double().cpu()
        same = (a == b) | (torch.isnan(a) & torch.isnan(b))
        off = (a - b).abs()
        ok = bool((same | (off <= tol)).all())
        assert ok, (what, float((off - tol)[~same].max()))

    if got.logprob is not None:
        w = want["logprob"]
        near(got.logprob, w, torch.where(torch.isfinite(w), 3 * U * w.abs() + 2 * U * math.log(vocab) + n, torch.zeros_like(w)), "logprob")
    near(got.entropy, want["entropy"], (n + 8 * U) * (1 + want["entropy"]), "entropy")
    near(got.norm[:, 0], want["norm"][:, 0], 0.0, "largest")
    near(got.norm[:, 1], want["norm"][:, 1], n * want["norm"][:, 1], "sum")
    if top:
        assert torch.equal(got.top_ids.long().cpu(), want["top_ids"])
        w = want["top_logprobs"]
        near(got.top_logprobs, w, torch.where(torch.isfinite(w), 3 * U * w.abs() + 2 * U * math.log(vocab) + n, torch.zeros_like(w)), "top")
    del far


VOCABS = [1, 2, 7, 10, 31, 32, 33, 64, 100, 255, 257, 500, 1000, 1024, 1025, 2047, 4097, 10000, 32768, 50001]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", VOCABS)
def test_rows_of_every_length(slaq, vocab, dtype):
    for rows, pad, scale, top in ((1, 0, 1.0, 5), (3, 1, 0.7, 32), (37, 8, 1.0 / 0.7, 1), (6, 3, 1.0, 0)):
        x, t, _ = _rows(rows, vocab, dtype, pad, vocab * 31 + rows)
        _check(slaq.token_logprobs(x, t, top=top, scale=scale), ref.logprobs(x, t, scale, top), vocab, x, scale, top)


@pytest.mark.parametrize("vocab,rows", [(130001, 2), (262144, 1), (1 << 20, 1)])
def test_long_rows(slaq, vocab, rows):
    for dtype in (torch.bfloat16, torch.float32):
        x, t, _ = _rows(rows, vocab, dtype, 5, vocab)
        _check(slaq.token_logprobs(x, t, top=20), ref.logprobs(x, t, 1.0, 20), vocab, x, 1.0, 20)


@pytest.mark.parametrize("vocab", [10, 700, 5000])
def test_many_rows(slaq, vocab):
    rows = 3001
    x, t, g = _rows(rows, vocab, torch.bfloat16, 0, 5)
    t[torch.randint(rows, (500,), generator=g).cuda()] = -1
    _check(slaq.token_logprobs(x, t, top=3), ref.logprobs(x, t, 1.0, 3), vocab, x, 1.0, 3)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [5, 40, 300, 3000, 40000])
def test_masks_infinities_and_rows_not_asked_for(slaq, vocab, dtype):
    x, t, g = _rows(16, vocab, dtype, 3, vocab)
    low, k = torch.finfo(dtype).min, vocab // 2
    x[1, k:] = -math.inf                 # half of the vocabulary is masked, by -inf or by the type's lowest value
    x[2, :k] = low
    x[3] = -math.inf                     # nothing is left
    x[4] = low                           # everything is masked alike: uniform
    x[5, k] = math.nan
    x[6, k] = math.inf
    x[7] = -math.inf
    x[7, vocab - 1] = 2.0                # one token is left
    x[8, 0] = -math.inf
    t[8] = 0                             # the given token is masked
    x[9] = 1.5                           # all equal
    x[10, k] = math.nan
    x[10, 0] = math.inf
    x[11] = -0.0
    x[11, vocab - 1] = 0.0               # equal to -0: the lower index stands first
    t[7] = vocab - 1
    t[12], t[13], t[14] = -1, -100, vocab
    x[13] = math.nan                     # not read
    t[15] = vocab + 5
    x[15] = -math.inf
    for scale in (1.0, 0.25):
        _check(slaq.token_logprobs(x, t, top=6, scale=scale), ref.logprobs(x, t, scale, 6), vocab, x, scale, 6)


@pytest.mark.parametrize("vocab", [50, 800, 9000, 70000])
@pytest.mark.parametrize("order", ["rising", "falling", "few values", "one block"])
def test_alternatives_in_awkward_orders(slaq, vocab, order):
    g = torch.Generator().manual_seed(vocab)
    ramp = torch.linspace(-4, 4, vocab)
    rows = {"rising": ramp, "falling": ramp.flip(0), "few values": torch.randint(3, (vocab,), generator=g).float(),
            "one block": torch.where(torch.arange(vocab) // 64 == vocab // 128, 5.0 + ramp, ramp * 0.1)}[order]
    x = rows[None, :].repeat(2, 1).to(torch.bfloat16).cuda()
    t = torch.zeros(2, dtype=torch.int64, device="cuda")
    for top in (1, 7, 32):
        _check(slaq.token_logprobs(x, t, top=top), ref.logprobs(x, t, 1.0, top), vocab, x, 1.0, top)


@pytest.mark.parametrize("vocab", [20, 900, 6000, 200000])
def test_rows_of_nan(slaq, vocab):
    x = torch.full((3, vocab), math.nan, dtype=torch.bfloat16, device="cuda")
    x[1, ::2] = 1.0
    x[2, : vocab - 3] = -math.inf
    t = torch.zeros(3, dtype=torch.int64, device="cuda")
    for top in (2, 7):
        got = slaq.token_logprobs(x, t, top=top)
        assert bool(got.logprob.isnan().all()) and bool(got.entropy.isnan().all()) and bool(got.top_logprobs.isnan().all())
        want = [list(range(top)), [2 * k + 1 for k in range(top)], ([vocab - 3, vocab - 2, vocab - 1] + list(range(top)))[:top]]
        assert got.top_ids.tolist() == want


@pytest.mark.parametrize("scale", [1e-38, 1e-6, 1e6, 1e30])
def test_extreme_temperatures(slaq, scale):
    """At a scale of 1e30 only the largest logit counts; at 1e-38 all are alike."""
    x, t, _ = _rows(5, 3000, torch.float32, 0, 3)
    _check(slaq.token_logprobs(x, t, top=4, scale=scale), ref.logprobs(x, t, scale, 4), 3000, x, scale, 4)


def test_without_targets_only_the_rows_themselves_are_described(slaq):
    x, t, _ = _rows(9, 1234, torch.bfloat16, 2, 1)
    got = slaq.token_logprobs(x, top=4)
    assert got.logprob is None
    _check(got, ref.logprobs(x, None, 1.0, 4), 1234, x, 1.0, 4)


def test_overlapping_and_repeated_rows(slaq):
    flat = torch.randn(4000, generator=torch.Generator().manual_seed(3)).cuda()
    x = flat.as_strided((7, 900), (450, 1))
    t = torch.arange(7, device="cuda")
    _check(slaq.token_logprobs(x, t, top=2), ref.logprobs(x, t, 1.0, 2), 900, x, 1.0, 2)
    x = flat[:900].expand(5, 900)
    _check(slaq.token_logprobs(x, t[:5], top=2), ref.logprobs(x, t[:5], 1.0, 2), 900, x, 1.0, 2)


def test_no_rows(slaq):
    got = slaq.token_logprobs(torch.empty(0, 50, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda"), top=3)
    assert got.logprob.numel() == 0 and got.top_ids.shape == (0, 3)


def test_results_do_not_change_from_call_to_call(slaq):
    x, t, _ = _rows(300, 20011, torch.bfloat16, 0, 9)
    a = slaq.token_logprobs(x, t, top=8)
    for _ in range(5):
        for p, q in zip(a, slaq.token_logprobs(x, t, top=8)):
            assert torch.equal(p, q)
    one = slaq.token_logprobs(x[17:18], t[17:18], top=8)     # nor much with the batch around a row
    torch.testing.assert_close(one.logprob, a.logprob[17:18], rtol=0, atol=(80 + 2 * 20011 / 256) * U)
    assert torch.equal(one.top_ids, a.top_ids[17:18])


def test_on_another_stream_and_in_a_graph(slaq):
    x, t, _ = _rows(40, 6001, torch.bfloat16, 0, 11)
    want = slaq.token_logprobs(x, t, top=5)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = slaq.token_logprobs(x, t, top=5, stream=side)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    got = slaq.token_logprobs(x, t, top=5, stream=side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    static = x.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = slaq.token_logprobs(static, t, top=5)
    for seed in (1, 2):
        y, _, _ = _rows(40, 6001, torch.bfloat16, 0, seed)
        static.copy_(y)
        graph.replay()
        want = slaq.token_logprobs(y, t, top=5)
        assert all(torch.equal(p, q) for p, q in zip(want, got))


def test_refusals(slaq):
    x, t, _ = _rows(4, 100, torch.float32, 0, 1)
    for call, code in ((lambda: slaq.token_logprobs(x, t, top=33), -2), (lambda: slaq.token_logprobs(x, t, top=-1), -1),
                       (lambda: slaq.token_logprobs(x, t, scale=0.0), -1), (lambda: slaq.token_logprobs(x, t, scale=math.inf), -1),
                       (lambda: slaq.token_logprobs(x, t, scale=-1.0), -1), (lambda: slaq.token_logprobs(x, t, scale=math.nan), -1),
                       (lambda: slaq.token_logprobs(x.double(), t), -1), (lambda: slaq.token_logprobs(x[0], t), -1),
                       (lambda: slaq.token_logprobs(x, t[:3]), -1), (lambda: slaq.token_logprobs(x, t.int()), -1),
                       (lambda: slaq.token_logprobs(x.t(), t[:1].expand(100)), -1), (lambda: slaq.token_logprobs(x.cpu(), t), -1),
                       (lambda: slaq.token_logprobs(x, t.cpu()), -1), (lambda: slaq.token_logprobs(x[:, :0], t), -1)):
        with pytest.raises(slaq.SlaqError) as e:
            call()
        assert e.value.code == code
