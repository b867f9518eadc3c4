"""Streams other than the current one: whose memory results and states are, and who waits for whom."""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def slaq():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_1802_04819_b200 as mod
    mod.build()
    return mod


def test_a_raw_stream_of_0_is_the_default_stream(slaq, monkeypatch):
    """torch takes a raw 0 for "no stream given" and makes another one, which is ordered behind nothing.  What stream a call runs on is
    seen by the call itself."""
    from paper_1802_04819_b200 import training
    x, t = torch.randn(4, 100, device="cuda"), torch.arange(4, device="cuda")
    plan = slaq.AdamW([x.clone()], [x])
    training._load()
    seen, current = [], training._current_stream
    monkeypatch.setattr(training, "_current_stream", lambda gpu: seen.append(current(gpu)) or seen[-1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for raw in (0, side.cuda_stream):
        with torch.cuda.stream(side):
            slaq.token_logprobs(x, t, stream=raw)
            plan.step(stream=raw)
        assert seen and set(seen) == {raw}
        seen.clear()
        torch.cuda.synchronize()


def test_appends_on_a_stream_that_lags_behind(slaq):
    """The losses are dropped at once and their size of memory is taken and written on the current stream, while the handle's stream has
    the append still before it: the histories are those of the same losses through the host."""
    jobs, rows_each = 50, 7
    rng = np.random.default_rng(2)
    ids = np.arange(jobs, dtype=np.int32)
    side = torch.cuda.Stream()
    d_ids, off = torch.arange(jobs, dtype=torch.int32, device="cuda"), torch.arange(jobs + 1, device="cuda") * rows_each
    targets = torch.zeros(jobs * rows_each, dtype=torch.int64, device="cuda")
    with slaq.Scheduler(jobs, 32, 8, stream=side) as a, slaq.Scheduler(jobs, 32, 8) as b:
        for s in (a, b):
            s.append_losses(ids, np.full(jobs, 5.0))
            s.set_time_model(ids, np.full(jobs, 0.1), np.full(jobs, 2.0))
        kept, want = [], []
        for k in range(10):
            lp = torch.from_numpy((-4.0 * 0.8 ** k * rng.uniform(0.9, 1.1, jobs * rows_each)).astype(np.float32)).cuda()
            want.append(slaq.job_losses(off, targets, lp).cpu().numpy())
            kept.append(lp)                                  # the inputs are the caller's to keep
        side.wait_stream(torch.cuda.current_stream())
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)                    # some ten milliseconds
        junk = []
        for lp in kept:
            a.append_token_losses(d_ids, off, targets, lp)
            junk.append(torch.full((jobs,), -1e9, dtype=torch.float64, device="cuda"))
        torch.cuda.synchronize()
        for losses in want:
            b.append_losses(ids, losses)
        np.testing.assert_array_equal(a.schedule(1.0, 100)[0], b.schedule(1.0, 100)[0])
        np.testing.assert_array_equal(a.get_predictions()["gain"], b.get_predictions()["gain"])
        assert all(bool((x == -1e9).all()) for x in junk)


@pytest.mark.parametrize("bits", [8, 32])
def test_a_plan_and_its_states_are_dropped_while_another_stream_steps(slaq, bits):
    """What is allocated in their place afterwards keeps its pattern, and the steps come out as if nothing had been dropped."""
    n = 3_000_000
    p, g = torch.ones(n, device="cuda"), torch.ones(n, device="cuda")
    plan = slaq.AdamW([p], [g], groups=[dict(lr=0.01, weight_decay=0.0)], state_bits=bits)
    sizes = [x.numel() * x.element_size() for xs in (plan.exp_avg, plan.exp_avg_sq, plan.exp_avg_scale or [], plan.exp_avg_sq_scale or [], [plan._ws]) for x in xs]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    for _ in range(20):
        plan.step(stream=side)
    del plan
    junk = [torch.full((size,), 85, dtype=torch.uint8, device="cuda") for size in sizes for _ in range(2)]
    torch.cuda.synchronize()
    assert all(bool((x == 85).all()) for x in junk)
    # 20 steps of lr, each off by the roundings of a step; 8-bit states: a constant gradient is the largest of its block, and kept exactly
    torch.testing.assert_close(p, torch.full_like(p, 0.8), rtol=0, atol=1e-4)


def test_a_cluster_of_training_jobs_on_another_stream(slaq):
    """The scheduler's handle and the trainers are on one stream, whichever is current."""
    from paper_1802_04819_b200 import trainers
    want, jobs = trainers.run("slaq", n_jobs=12, epochs=6)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got, others = trainers.run("slaq", n_jobs=12, epochs=6)
        torch.cuda.synchronize()
    assert got == want and torch.equal(jobs.weights, others.weights)
