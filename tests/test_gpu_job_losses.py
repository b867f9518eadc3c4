"""Mean losses of jobs and the rows' factors in them, and the append that takes them into the histories.  Sums are of 64-bit
terms (products of fp32 numbers are exact): a loss is within (rows + 4) 2^-53 of the sum of the terms' sizes; factors are one rounding."""

import math

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


def _inputs(lengths, seed, weighted, missing, behind=3):
    g = torch.Generator().manual_seed(seed)
    off = torch.zeros(len(lengths) + 1, dtype=torch.int64)
    off[1:] = torch.tensor(lengths, dtype=torch.int64).cumsum(0)
    rows = int(off[-1]) + behind
    t = torch.where(torch.rand(rows, generator=g) < missing, torch.tensor(-1), torch.tensor(5))
    lp = -3 * torch.rand(rows, generator=g)
    w = torch.rand(rows, generator=g) * (torch.rand(rows, generator=g) < 0.9) if weighted else None
    return off, t, lp, w


CASES = [[1], [0], [300_001], [140_000, 3, 130_000], [4] * 200 + [2049, 0, 30_000, 2048] + [3] * 300, [3, 0, 0, 5], [1] * 700, [31, 32, 33, 255, 256, 257, 0, 1023, 1025], [70001], [5, 200003, 0, 1, 4096], [9] * 3000, [120] * 148]


@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("lengths", CASES, ids=lambda v: f"{len(v)}x{max(v)}")
def test_losses_and_factors(slaq, lengths, weighted):
    off, t, lp, w = _inputs(lengths, len(lengths), weighted, 0.2)
    cuda = lambda v: None if v is None else v.cuda()   # noqa: E731
    want, factors = ref.job_losses(off.tolist(), t.tolist(), lp, w)
    got = slaq.job_losses(cuda(off), cuda(t), cuda(lp), cuda(w)).cpu()
    for j, n in enumerate(lengths):
        if math.isnan(want[j]):
            assert math.isnan(got[j])
        else:
            assert abs(float(got[j] - want[j])) <= (n + 4) * 2.0 ** -53 * 4 * 3
    out = torch.full((len(lp),), 9.0).cuda()
    got = slaq.job_row_grad(cuda(off), cuda(t), cuda(w), out=out).cpu().double()
    end = int(off[-1])
    assert bool((got[end:] == 9.0).all())                                  # rows behind the last job stay as they were
    assert bool(((got[:end] - factors[:end]).abs() <= (2.0 ** -24 + 1e-12) * factors[:end].abs()).all())
    off2 = off + 3                                                          # rows in front as well: zeros in a result of its own
    pad = lambda v, x: None if v is None else torch.cat([torch.full((3,), x, dtype=v.dtype), v]).cuda()   # noqa: E731
    fresh = slaq.job_row_grad(off2.cuda(), pad(t, 5), pad(w, 1.0)).cpu().double()
    assert not fresh[:3].any() and not fresh[3 + end:].any() and torch.equal(fresh[3:3 + end], got[:end])
    again = slaq.job_losses(cuda(off), cuda(t), cuda(lp), cuda(w)).cpu()
    assert torch.equal(torch.nan_to_num(again), torch.nan_to_num(slaq.job_losses(cuda(off), cuda(t), cuda(lp), cuda(w)).cpu()))


def test_offsets_that_leave_the_rows_touch_nothing(slaq):
    off = torch.tensor([0, 4, 2, 6, 99, 99, 10], device="cuda")            # falls; ends behind the rows
    lp, out = -torch.ones(10, device="cuda"), torch.full((10,), 9.0, device="cuda")
    loss = slaq.job_losses(off, None, lp).cpu()
    assert [math.isnan(v) for v in loss.tolist()] == [False, True, False, True, True, True]
    slaq.job_row_grad(off, out=out)
    np.testing.assert_array_equal(out.cpu().numpy(), np.float32([-.25, -.25, -.25, -.25, -.25, -.25, 9, 9, 9, 9]))
    for bad in ([-3, 2], [-(2 ** 62), 2 ** 62], [0, 2 ** 40], [11, 12]):
        assert math.isnan(float(slaq.job_losses(torch.tensor(bad, device="cuda"), None, lp)))


def test_masked_tokens_count_only_where_they_have_weight(slaq):
    lp = torch.tensor([-1.0, -math.inf, -2.0, math.nan, -3.0], device="cuda")
    w = torch.tensor([1.0, 0.0, 1.0, 0.0, 2.0], device="cuda")
    off = torch.tensor([0, 5], device="cuda")
    assert float(slaq.job_losses(off, None, lp, w)) == 2.25
    assert float(slaq.job_losses(off, None, lp)) != float(slaq.job_losses(off, None, lp))    # NaN counts there
    t = torch.tensor([0, -1, 0, -1, 0], device="cuda")
    assert float(slaq.job_losses(off, t, lp)) == 2.0


def test_the_scheduler_takes_them_as_the_jobs_losses(slaq):
    jobs = 40
    rng = np.random.default_rng(3)
    lengths = rng.integers(1, 60, jobs)
    off, t, lp, w = _inputs(lengths.tolist(), 1, True, 0.0, behind=0)
    w = w + 0.1
    ids = np.arange(jobs, dtype=np.int32)
    d_ids = torch.arange(jobs, dtype=torch.int32, device="cuda")
    times = torch.full((jobs,), 2.0, dtype=torch.float64, device="cuda")
    with slaq.Scheduler(jobs, 32, 8) as a, slaq.Scheduler(jobs, 32, 8) as b:
        for s in (a, b):
            s.append_losses(ids, np.full(jobs, 5.0), np.full(jobs, 2.0))
        for k in range(8):
            lp_k = (lp * 0.8 ** k).cuda()
            got = a.append_token_losses(d_ids, off.cuda(), t.cuda(), lp_k, w.cuda(), d_iter_times=times)
            want = slaq.job_losses(off.cuda(), t.cuda(), lp_k, w.cuda())
            assert torch.equal(got, want)
            b.append_losses(ids, want.cpu().numpy(), np.full(jobs, 2.0))
        x, y = a.schedule(3.0, 100), b.schedule(3.0, 100)
        np.testing.assert_array_equal(x[0], y[0])
        np.testing.assert_array_equal(a.get_predictions()["gain"], b.get_predictions()["gain"])
        # a job whose rows all have no weight has no loss: skipped, and the next epoch says so
        a.append_token_losses(d_ids[:2], torch.tensor([0, 3, 6], device="cuda"), None, lp.cuda()[:6], torch.tensor([1., 1, 1, 0, 0, 0], device="cuda"))
        with pytest.raises(slaq.SlaqError, match="skipped"):
            a.schedule(3.0, 100)
        a.schedule(3.0, 100)


def test_refusals(slaq):
    lp = -torch.ones(10, device="cuda")
    off = torch.tensor([0, 10], device="cuda")
    t = torch.zeros(10, dtype=torch.int64, device="cuda")
    with slaq.Scheduler(4, 8, 4) as s:
        for call in (lambda: slaq.job_losses(off.int(), t, lp), lambda: slaq.job_losses(off, t[:9], lp), lambda: slaq.job_losses(off, t, lp.double()),
                     lambda: slaq.job_losses(off[:0], t, lp), lambda: slaq.job_row_grad(off), lambda: slaq.job_losses(off, t, lp, out=lp),
                     lambda: s.append_token_losses(torch.zeros(2, dtype=torch.int32, device="cuda"), off, t, lp),
                     lambda: s.append_token_losses(torch.zeros(1, dtype=torch.int64, device="cuda"), off, t, lp),
                     lambda: s.append_token_losses(torch.zeros(5, dtype=torch.int32, device="cuda"), torch.tensor([0, 1, 2, 3, 4, 5], device="cuda"), t, lp)):
            with pytest.raises(slaq.SlaqError) as e:
                call()
            assert e.value.code == -1
