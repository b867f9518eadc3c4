"""Matrices, strides and tensors that 32-bit positions do not reach, checked at their far ends."""

import pytest
import torch

import token_rows as ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
ROWS, VOCAB = 16_500, 131_072                 # 2^31 is passed in row 16,384


@pytest.fixture(scope="module")
def slaq():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_1802_04819_b200 as mod
    mod.build()
    yield mod
    torch.cuda.empty_cache()


def _check(x, t, g, logprob, grad, where, want_x):
    """Log probabilities as in test_gpu_token_logprobs, gradients within their own rounding to bf16 and the probabilities' error."""
    want = ref.logprobs(want_x, t)
    n = (40 + want_x.shape[1] / 256) * U
    off = (logprob.double().cpu() - want["logprob"]).abs()
    assert bool((off <= 3 * U * want["logprob"].abs() + 30 * U + n).all()), where
    dx = ref.gradient(want_x, t, g)
    off = (grad.double().cpu() - dx).abs()
    assert bool((off <= 2.0 ** -8 * dx.abs() + 64 * U * float(g[0].abs()) + 2.0 ** -133).all()), where


def test_a_matrix_of_more_than_2_to_the_31_elements(slaq):
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(ROWS, VOCAB, dtype=torch.bfloat16, device="cuda")
    for lo in range(0, ROWS, 500):
        x[lo: lo + 500] = 2 * torch.randn(500, VOCAB, generator=gen, device="cuda")
    t = torch.randint(VOCAB, (ROWS,), generator=gen, device="cuda")
    g = torch.full((ROWS,), -0.5, device="cuda")
    far = torch.tensor([0, 16_383, 16_384, 16_385, ROWS - 1])
    kept = x[far.cuda()].cpu()
    r = slaq.token_logprobs(x, t, top=3)
    for i, k in enumerate(far.tolist()):
        best = torch.argsort(-kept[i].double(), stable=True)[:3]
        assert r.top_ids[k].tolist() == best.tolist()
    apart = torch.empty_like(x)
    slaq.token_logprobs_grad(x, t, r.norm, g, out=apart)
    _check(x, t[far.cuda()].cpu(), g.cpu(), r.logprob[far.cuda()], apart[far.cuda()], "gradient", kept)
    del apart
    logprob, grad = slaq.token_loss(x, t, g, out=x)
    _check(x, t[far.cuda()].cpu(), g.cpu(), logprob[far.cuda()], grad[far.cuda()], "in place", kept)


def test_rows_that_are_2_to_the_30_elements_apart(slaq):
    gen = torch.Generator(device="cuda").manual_seed(2)
    pitch = 2 ** 30 + 8
    flat = torch.zeros(3 * pitch + 5001, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(flat, (4, 5001), (pitch, 1))
    x.copy_(2 * torch.randn(4, 5001, generator=gen, device="cuda"))
    kept, t, g = x.cpu(), torch.randint(5001, (4,), generator=gen, device="cuda"), torch.full((4,), -0.25, device="cuda")
    logprob, grad = slaq.token_loss(x, t, g)
    _check(x, t.cpu(), g.cpu(), logprob, grad, "apart", kept)
    logprob, grad = slaq.token_loss(x, t, g, out=x)
    _check(x, t.cpu(), g.cpu(), logprob, grad, "in place", kept)
    assert not flat[5001: pitch].any() and not flat[pitch + 5001: pitch + 10_000].any()


@pytest.mark.parametrize("bits", [8, 32])
def test_a_tensor_of_more_than_2_to_the_31_elements(slaq, bits):
    """Blocks of 256 elements do not know of one another: the last ones are those of a small tensor."""
    n, tail = 2 ** 31 + 1003, 256 * 40 + 1003
    gen = torch.Generator(device="cuda").manual_seed(3)
    p, g = (torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    p[-tail:], g[-tail:] = torch.randn(tail, generator=gen, device="cuda"), 0.1 * torch.randn(tail, generator=gen, device="cuda")
    q, h = p[-tail:].clone(), g[-tail:].clone()
    large, small = slaq.AdamW([p], [g], groups=[dict(lr=0.01)], state_bits=bits), slaq.AdamW([q], [h], groups=[dict(lr=0.01)], state_bits=bits)
    for _ in range(2):
        large.step()
        small.step()
    assert torch.equal(p[-tail:], q) and not p[: 2 ** 20].any()
    for a, b in ((large.exp_avg, small.exp_avg), (large.exp_avg_sq, small.exp_avg_sq)):
        assert torch.equal(a[0][-tail:].view(torch.uint8), b[0].view(torch.uint8))
    if bits == 8:
        assert torch.equal(large.exp_avg_scale[0][-44:], small.exp_avg_scale[0]) and torch.equal(large.exp_avg_sq_scale[0][-44:], small.exp_avg_sq_scale[0])
