"""Every iteration of training jobs, weights, moments and gradients, against 64 bits.

The step is held to the formula from the gradient that the GPU computed (tolerances of test_gpu_adamw), the gradient to its own formula from
the weights that the GPU had.  For the gradient, u = 2^-24: a logit is a sum of F products, off by (F + 1) u sum |x w|; a
probability by twice the row's largest such error and 20 u of itself (exponential, sum of 5, division); the factor 1 / rows by u;
the sum over R rows adds (R + 3) u of the terms' sizes."""

import pytest
import torch

from test_gpu_adamw import _check_32

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("idle", [False, True])
def test_every_iteration(idle):
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_1802_04819_b200 as slaq
    slaq.build()
    from paper_1802_04819_b200.trainers import SoftmaxJobs
    J, R, F, C = 4, 50, 6, 5
    jobs = SoftmaxJobs(J, rows=R, features=F, classes=C, seed=9)
    x, labels = jobs.x.double().cpu(), jobs.labels.cpu().view(J, R)
    one = torch.nn.functional.one_hot(labels, C).double()
    rates, taken = [g["lr"] for g in jobs.adamw._groups], [0] * J
    for k in range(6):
        old_w = jobs.weights.cpu().clone()
        old_m, old_v = ([t.cpu().clone() for t in ts] for ts in (jobs.adamw.exp_avg, jobs.adamw.exp_avg_sq))
        active = torch.tensor([1, 0, k % 2, 3], dtype=torch.int32, device="cuda") if idle else None
        jobs.step(active=active)
        w = old_w.double()
        p = torch.softmax(torch.bmm(x, w), 2)
        grad = torch.bmm(x.transpose(1, 2), (p - one) / R)
        logit = (F + 1) * U * torch.bmm(x.abs(), w.abs()).amax(2, keepdim=True)
        term = (p * (2 * logit + 20 * U) + ((R + 3) * U + U) * (p - one).abs()) / R
        room = torch.bmm(x.abs().transpose(1, 2), term)
        assert bool(((jobs.grads.double().cpu() - grad).abs() <= room).all())
        for j in range(J):
            if idle and int(active[j]) <= 0:
                assert torch.equal(jobs.weights[j].cpu(), old_w[j]) and torch.equal(jobs.adamw.exp_avg[j].cpu(), old_m[j])
                continue
            h = dict(lr=rates[j], betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0, step=taken[j])
            _check_32(jobs.weights[j].flatten(), jobs.adamw.exp_avg[j].flatten(), jobs.adamw.exp_avg_sq[j].flatten(), old_w[j].flatten(),
                      jobs.grads[j].cpu().flatten(), old_m[j].flatten(), old_v[j].flatten(), h, torch.float32)
            taken[j] += 1
    assert jobs.adamw.get_steps().tolist() == taken
