"""Training jobs on the scheduler's GPU: multinomial logistic regression, one of the algorithms of the paper's cluster experiment
(Evaluation, "Experimental setup"), many jobs trained side by side with the operators of ``training``.

Each job has its own data (seeded, drawn: the paper's datasets are not available), weights, learning rate and AdamW group, and reports
the mean cross entropy over its rows once per iteration.  The losses are those of real optimisation runs, not draws
from the two curve families, which is what the paper's prediction error is about.

    python -m paper_1802_04819_b200.trainers            # needs a GPU; a cluster of such jobs, scheduled and by fair share
"""

from __future__ import annotations

import math

import numpy as np


class SoftmaxJobs:
    """``n_jobs`` jobs of ``rows`` examples, ``features`` features (a constant one among them) and ``classes`` classes.  Labels
    follow a random linear model with noise; learning rates are drawn log-uniform from ``rates``."""

    def __init__(self, n_jobs, rows=256, features=24, classes=10, rates=(2e-3, 5e-2), noise=1.0, state_bits=32, seed=0):
        import torch

        from .training import AdamW, job_row_grad
        g = torch.Generator(device="cuda").manual_seed(seed)
        draw = lambda *shape: torch.randn(*shape, generator=g, device="cuda")   # noqa: E731
        self.n_jobs, self.rows, self.classes = n_jobs, rows, classes
        self.x = draw(n_jobs, rows, features)
        self.x[:, :, 0] = 1.0
        score = torch.bmm(self.x, draw(n_jobs, features, classes)) + noise * draw(n_jobs, rows, classes)
        self.labels = score.argmax(2).flatten()
        self.offsets = torch.arange(n_jobs + 1, device="cuda") * rows
        self.weights = torch.zeros(n_jobs, features, classes, device="cuda")
        self.grads = torch.zeros_like(self.weights)
        self.row_grad = job_row_grad(self.offsets, self.labels)
        rate = torch.exp(math.log(rates[0]) + math.log(rates[1] / rates[0]) * torch.rand(n_jobs, generator=g, device="cuda")).tolist()
        self.adamw = AdamW(list(self.weights), list(self.grads), range(n_jobs), [dict(lr=r, weight_decay=0.0) for r in rate], state_bits=state_bits)

    def step(self, active=None, losses=None):
        """One iteration of the jobs with an entry above 0 in ``active`` (int32 [n_jobs]; None: all).  Returns every job's loss before it
        (float64 [n_jobs] on the GPU)."""
        import torch

        from .training import job_losses, token_loss
        logits = torch.bmm(self.x, self.weights).view(-1, self.classes)
        logprob, grad = token_loss(logits, self.labels, self.row_grad, out=logits)
        torch.bmm(self.x.transpose(1, 2), grad.view(self.n_jobs, self.rows, self.classes), out=self.grads)
        losses = job_losses(self.offsets, self.labels, logprob, out=losses)
        self.adamw.step(active)
        return losses

    def histories(self, iterations):
        """The losses of every job's next iterations, float64 [n_jobs, iterations] on the host."""
        import torch
        out = torch.empty(iterations, self.n_jobs, dtype=torch.float64, device="cuda")
        for k in range(iterations):
            self.step(losses=out[k])
        return out.t().contiguous().cpu().numpy()


def run(policy="slaq", n_jobs=64, epochs=80, total_cores=64, max_cores_per_job=16, epoch_seconds=3.0, max_hist=64, seed=0):
    """A cluster of such jobs, which arrive one after the other over three quarters of the epochs.  In an epoch a job on n cores finishes
    the iterations that its law t(n) = s + w/n allows (drawn laws; the jobs themselves run on this GPU).  "fair": the cores in
    equal parts.  Returns the loss averaged over the running jobs and the epochs, each job's normalised by its first loss and the
    lowest that it reaches when it is trained to the end, and the jobs."""
    import torch

    import paper_1802_04819_b200 as slaq
    rng = np.random.default_rng(seed)
    s, w = rng.uniform(0.05, 0.5, n_jobs), rng.uniform(1.0, 20.0, n_jobs)
    last = SoftmaxJobs(n_jobs, seed=seed).histories(400).min(axis=1)
    jobs = SoftmaxJobs(n_jobs, seed=seed)
    nobody = torch.zeros(n_jobs, dtype=torch.int32, device="cuda")
    first = jobs.step(active=nobody).cpu().numpy()
    arrives = np.arange(n_jobs) * (0.75 * epochs) / n_jobs
    credit, mean = np.zeros(n_jobs), []
    with slaq.Scheduler(n_jobs, max_hist, max_cores_per_job, stream=torch.cuda.current_stream()) as sched:   # the losses are made there
        for epoch in range(epochs):
            new = np.nonzero(np.ceil(arrives) == epoch)[0]
            if new.size:
                sched.append_losses(new, first[new])
                sched.set_time_model(new, s[new], w[new])
            running = arrives <= epoch
            if policy == "slaq":
                alloc, _ = sched.schedule(epoch_seconds, total_cores)
            else:
                alloc = np.where(running, min(max_cores_per_job, total_cores // int(running.sum())), 0)
                alloc[np.nonzero(running)[0][: max(0, total_cores - int(alloc.sum()))]] += int(alloc.max()) < max_cores_per_job
            progress = np.where(alloc > 0, epoch_seconds / (s + w / np.maximum(alloc, 1)), 0.0) + credit
            todo = np.floor(progress).astype(np.int32)
            credit = progress - todo
            left = torch.from_numpy(todo).cuda()
            for k in range(1, int(todo.max()) + 1):
                jobs.step(active=left)
                left -= 1
                losses = jobs.step(active=nobody)
                ran = torch.nonzero((left >= 0) & (torch.from_numpy(todo).cuda() > 0)).flatten().to(torch.int32)
                sched.append_losses_device(ran, losses[ran.long()])
            now = jobs.step(active=nobody).cpu().numpy()
            mean.append(float(np.mean(((now - last) / (first - last))[running])))
    return float(np.mean(mean)), jobs


if __name__ == "__main__":
    import json
    print(json.dumps({policy: run(policy)[0] for policy in ("slaq", "fair")}))
