"""The trainers' operators as they are used together: jobs that train under the scheduler."""

import numpy as np
import pytest
import torch

import token_rows as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def slaq():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_1802_04819_b200 as mod
    mod.build()
    return mod


@pytest.mark.parametrize("state_bits", [32, 8])
def test_iterations_are_those_of_64_bits(slaq, state_bits):
    """Three iterations of a few jobs against the formulas in 64 bits.  With states in 32 bits an iteration's rounding, 2^-24
    of sums over 50 rows and 6 features, is far below 1e-5 of a loss of about 2; AdamW divides a gradient by its own size, so where
    one is near 0 that rounding counts whole: a weight is compared where its gradient is above 1e-4.  With 8 bits the
    first iteration knows nothing of the states' rounding."""
    from paper_1802_04819_b200.trainers import SoftmaxJobs
    jobs = SoftmaxJobs(3, rows=50, features=6, classes=5, state_bits=state_bits, seed=4)
    x, labels = jobs.x.double().cpu(), jobs.labels.cpu().view(3, 50)
    w = jobs.weights.double().cpu()
    m, v = torch.zeros_like(w), torch.zeros_like(w)
    rates = [g["lr"] for g in jobs.adamw._groups]
    for k in range(3 if state_bits == 32 else 1):
        losses = jobs.step().cpu()
        logits = torch.bmm(x, w)
        lp = torch.log_softmax(logits, 2).gather(2, labels[:, :, None])[:, :, 0]
        torch.testing.assert_close(losses, -lp.mean(1), rtol=1e-5, atol=0)
        one = torch.nn.functional.one_hot(labels, 5).double()
        grad = torch.bmm(x.transpose(1, 2), (torch.softmax(logits, 2) - one) / 50)
        torch.testing.assert_close(jobs.grads.double().cpu(), grad, rtol=0, atol=1e-5 if k else 1e-6)
        for j in range(3):
            w[j], m[j], v[j] = ref.adamw(w[j], grad[j], m[j], v[j], rates[j], (0.9, 0.999), 1e-8, 0.0, k)
        clear = grad.abs() > 1e-4
        if k == 0:
            torch.testing.assert_close(jobs.weights.double().cpu()[clear], w[clear], rtol=1e-3, atol=1e-6)
        w = jobs.weights.double().cpu()       # from here on as the jobs have it
        if state_bits == 32:
            m, v = (torch.stack([t.double().cpu().view(6, 5) for t in ts]) for ts in (jobs.adamw.exp_avg, jobs.adamw.exp_avg_sq))


def test_jobs_without_cores_do_not_move(slaq):
    from paper_1802_04819_b200.trainers import SoftmaxJobs
    jobs = SoftmaxJobs(6, rows=40, features=5, classes=3, seed=1)
    jobs.step()
    before = jobs.weights.clone()
    jobs.step(active=torch.tensor([1, 0, 4, 0, 0, 1], dtype=torch.int32, device="cuda"))
    moved = (jobs.weights != before).flatten(1).any(1).cpu().numpy()
    np.testing.assert_array_equal(moved, [True, False, True, False, False, True])
    np.testing.assert_array_equal(jobs.adamw.get_steps(), [2, 1, 2, 1, 1, 2])


def test_the_allocation_says_who_trains(slaq):
    """append_token_losses, schedule_device and the step in one stream, the allocation being the step's `active`: no host in between."""
    from paper_1802_04819_b200.training import token_loss
    from paper_1802_04819_b200.trainers import SoftmaxJobs
    n = 24
    jobs = SoftmaxJobs(n, rows=64, features=8, classes=4, seed=2)
    ids = torch.arange(n, dtype=torch.int32, device="cuda")
    alloc = torch.ones(n, dtype=torch.int32, device="cuda")
    with slaq.Scheduler(n, 32, 8) as sched:
        sched.append_losses(np.arange(n), jobs.step().cpu().numpy())
        sched.set_time_model(np.arange(n), np.full(n, 0.1), np.full(n, 2.0))
        total, cores = np.zeros(n, np.int64), []
        for _ in range(12):
            logits = torch.bmm(jobs.x, jobs.weights).view(-1, 4)
            logprob, grad = token_loss(logits, jobs.labels, jobs.row_grad)
            sched.append_token_losses(ids, jobs.offsets, jobs.labels, logprob)
            sched.schedule_device(1.0, n // 2, alloc)                         # fewer cores than jobs: no floor, some get several
            torch.bmm(jobs.x.transpose(1, 2), grad.view(n, 64, 4), out=jobs.grads)
            jobs.adamw.step(alloc)
            total += (alloc > 0).cpu().numpy()
            cores.append(int(alloc.sum()))
        np.testing.assert_array_equal(jobs.adamw.get_steps(), 1 + total)
        assert cores == [n // 2] * 12 and total.sum() > 0
        sched.schedule(1.0, n)                                                # nothing was skipped


def test_the_commands_run(slaq):
    from paper_1802_04819_b200 import accuracy, trainers
    r = accuracy.measure_trained(n_jobs=40, hmax=60)
    assert 0 < r["fitted"] <= 40 and np.isfinite(r["median_error"])
    for policy in ("slaq", "fair"):
        value, jobs = trainers.run(policy, n_jobs=8, epochs=4)
        assert np.isfinite(value) and int(jobs.adamw.get_steps().sum()) > 0
