"""Draws, losses, norms and steps together, as jobs on the scheduler's GPU run them.

Gradients against the formula in 64 bits: a product of `rows` terms, each rounded twice, in 32 bits: rows u of the sum of their sizes and 8u for the
probabilities (u = 2^-24)."""

import numpy as np
import pytest
import torch

import sampling
from test_gpu_adamw import _check_32

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def trainers():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    torch.backends.cuda.matmul.allow_tf32 = False
    import paper_1802_04819_b200 as mod
    mod.build()
    from paper_1802_04819_b200 import trainers
    return trainers


def _gradient(x, logits, answers, row_grad, temperature):
    """By the weights, in 64 bits, and the sum of its terms' sizes."""
    p = torch.softmax(logits.double() / temperature, 1)
    one = torch.zeros_like(p)
    one[torch.arange(p.shape[0]), answers] = 1.0
    by_logits = row_grad.double()[:, None] * (one - p) / temperature
    return x.double().t() @ by_logits, x.double().abs().t() @ (row_grad.double().abs()[:, None] * (one + p) / temperature)


@pytest.mark.parametrize("max_norm", [None, 0.05])
def test_jobs_that_learn_from_rewards(trainers, max_norm):
    jobs = trainers.RewardedJobs(7, rows=60, features=5, classes=6, temperature=0.8, max_norm=max_norm, rates=(1e-2, 1e-2))
    jobs.weights.normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    for _ in range(3):
        old = jobs.weights.cpu().clone()
        m, v = [t.cpu().clone() for t in jobs.adamw.exp_avg], [t.cpu().clone() for t in jobs.adamw.exp_avg_sq]
        steps = jobs.adamw.get_steps()
        logits = torch.bmm(jobs.x, jobs.weights).cpu()
        active = torch.tensor([1, 0, 2, 1, 1, 0, 1], dtype=torch.int32, device="cuda")
        wrong = jobs.step(active)
        labels, answers, u = jobs.labels.cpu().view(7, -1), jobs.answers.token.cpu().view(7, -1), jobs.uniform.cpu().view(7, -1)
        grads = jobs.grads.cpu()
        for j in range(7):
            want = [sampling.draw(logits[j, r].double().numpy(), float(u[j, r]), jobs.temperature)[0] for r in range(60)]
            assert answers[j].tolist() == want
            right = (answers[j] == labels[j]).float()
            assert abs(float(wrong[j]) - (1 - float(right.double().mean()))) <= 2 * U
            row_grad = (right.mean() - right) / 60
            g, size = _gradient(jobs.x[j].cpu(), logits[j], answers[j], row_grad, jobs.temperature)
            assert bool(((grads[j].double() - g).abs() <= (60 + 8) * U * size + 1e-12).all())
            norm = float(grads[j].double().square().sum().sqrt())
            factor = 1.0 if max_norm is None or norm <= max_norm else float(np.float32(max_norm / norm))
            if not int(active[j]):
                assert torch.equal(jobs.weights[j].cpu(), old[j])
                continue
            # a factor is off by 7u at most: as much of the gradient, which the bounds of the step leave room for by its size
            h = dict(lr=1e-2, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0, step=int(steps[j]), grad_scale=factor)
            if max_norm is not None:
                got = float(jobs.norms.measure(max_norm).factor[j])
                assert abs(got - factor) <= 8 * U * factor
                h["grad_scale"] = got
            _check_32(jobs.weights[j].flatten(), jobs.adamw.exp_avg[j].flatten(), jobs.adamw.exp_avg_sq[j].flatten(), old[j].flatten(), grads[j].flatten(),
                      m[j].flatten(), v[j].flatten(), h, torch.float32)


def test_clipped_jobs_without_a_limit_are_the_others(trainers):
    plain, clipped = (trainers.SoftmaxJobs(20, rows=50, max_norm=m) for m in (None, 1e9))
    for _ in range(4):
        assert torch.equal(plain.step(), clipped.step())
    assert torch.equal(plain.weights, clipped.weights)


def test_a_whole_step_in_a_graph(trainers):
    """Draw, score, norms and step, captured once and replayed, against the same calls one by one."""
    import paper_1802_04819_b200 as slaq
    g = torch.Generator().manual_seed(2)
    rows, vocab = 40, 3000
    w = torch.randn(16, vocab, generator=g)
    x = torch.randn(rows, 16, generator=g).cuda()

    def build():
        weights = w.clone().cuda()
        grads = torch.zeros_like(weights)
        return weights, grads, slaq.AdamW([weights], [grads], groups=[dict(lr=1e-2)]), slaq.GradNorms([grads])

    uniform = torch.rand(5, rows, generator=g).cuda()

    def step(state, u):
        weights, grads, adamw, norms = state
        logits = x @ weights
        drawn = slaq.sample_tokens(logits, u, 0.9, top_k=50, top_p=0.95)
        _, grad = slaq.token_loss(logits, drawn.token, row_grad, scale=1 / 0.9, out=logits)
        torch.mm(x.t(), grad, out=grads)
        norm, factor = norms.measure(0.1)
        adamw.step(factors=factor)
        return drawn.token, norm

    row_grad = torch.full((rows,), -1.0 / rows, device="cuda")
    one, two = build(), build()
    u = torch.empty(rows, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        spare = build()
        u.copy_(uniform[0])
        step(spare, u)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        token, norm = step(one, u)
    for k in range(5):
        u.copy_(uniform[k])
        graph.replay()
        want = step(two, uniform[k])
        assert torch.equal(token, want[0]) and torch.equal(norm, want[1])
    assert torch.equal(one[0], two[0])
