"""The factors of rows whose jobs are refused, in a result that the call makes itself: every row has one value, whatever the offsets."""

import pytest
import torch

pytestmark = pytest.mark.gpu

# offsets, and the factor of each row, of ten: 0 where no job counts it
CASES = [([0, 4, 2, 6, 99, 99, 10], [-1 / 4] * 6 + [0] * 4), ([0, 10, 11], [-1 / 10] * 10), ([-1, 3, 7], [0] * 3 + [-1 / 4] * 4 + [0] * 3),
         ([2, 5, 99], [0] * 2 + [-1 / 3] * 3 + [0] * 5), ([99, 0], [0] * 10), ([-4, 99], [0] * 10), ([5, 2, 8], [0] * 2 + [-1 / 6] * 6 + [0] * 2),
         ([0, 8, 3], [-1 / 8] * 8 + [0] * 2), ([6, 9, 1, 3], [0, -1 / 2, -1 / 2, 0, 0, 0] + [-1 / 3] * 3 + [0])]


@pytest.fixture(scope="module")
def slaq():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_1802_04819_b200 as mod
    mod.build()
    return mod


@pytest.mark.parametrize("scale", [1, 200, 2000, 40_000])       # a warp, a block of 128 or 512 threads, a cluster for each job
@pytest.mark.parametrize("offsets,factors", CASES, ids=lambda v: "-".join(map(str, v)) if isinstance(v[0], int) and len(v) < 9 else "")
def test_rows_of_refused_jobs_are_zeros(slaq, offsets, factors, scale):
    off = torch.tensor(offsets, device="cuda") * scale
    targets = torch.zeros(10 * scale, dtype=torch.int64, device="cuda")
    want = torch.tensor(factors, dtype=torch.float64).repeat_interleave(scale).div(scale)
    for _ in range(3):
        held = torch.full((10 * scale,), 9.0, device="cuda")     # what the result's memory held
        del held
        got = slaq.job_row_grad(off, targets).double().cpu()
        assert bool(((got - want).abs() <= 2.0 ** -24 * want.abs()).all())


@pytest.mark.parametrize("jobs,scale", [(5, 1), (2890, 1), (2900, 1), (30_000, 1), (5, 500), (720, 500), (730, 500), (3000, 200)])
def test_many_jobs_of_which_some_are_refused(slaq, jobs, scale):
    """Groups of five jobs with 3, 0, 4, 1 and 2 times so many rows; every seventh group's third offset leaves the array, so that two jobs
    are refused.  Zeros are written by the same kernel or, for more jobs, by one of their own."""
    lengths = torch.tensor([3, 0, 4, 1, 2]).repeat(jobs // 5) * scale
    off = torch.zeros(jobs + 1, dtype=torch.int64)
    off[1:] = lengths.cumsum(0)
    off += 6
    rows = int(off[-1]) + 5
    owner = torch.full((rows,), -1)
    owner[6: rows - 5] = torch.repeat_interleave(torch.arange(jobs), lengths)
    bad = torch.arange(2, jobs, 35)
    off[bad] = torch.where(bad % 2 == 0, torch.tensor(2 ** 40), torch.tensor(-7))
    refused = torch.zeros(jobs, dtype=torch.bool)
    refused[bad], refused[bad - 1] = True, True
    want = torch.where((owner < 0) | refused[owner], 0.0, -1.0 / lengths[owner].clamp_min(1).double())
    targets = torch.zeros(rows, dtype=torch.int64, device="cuda")
    held = torch.full((rows,), 9.0, device="cuda")
    del held
    got = slaq.job_row_grad(off.cuda(), targets).double().cpu()
    assert bool(((got - want).abs() <= 2.0 ** -24 * want.abs()).all())


@pytest.mark.parametrize("jobs", [2, 600, 3000])
def test_the_same_in_a_replayed_graph(slaq, jobs):
    off = torch.arange(0, 3 * jobs + 3, 3)
    rows = 3 * jobs + 4
    targets = torch.zeros(rows, dtype=torch.int64, device="cuda")
    d_off = off.cuda()
    slaq.job_row_grad(d_off, targets)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = slaq.job_row_grad(d_off, targets)
    for last in (2 ** 33, 3 * jobs + 1, 3 * jobs - 3):
        d_off[-1] = last
        got.fill_(9.0)
        graph.replay()
        want = torch.full((rows,), -1 / 3)
        want[3 * jobs - 3:] = 0.0
        if last == 3 * jobs + 1:
            want[3 * jobs - 3: last] = -1 / 4
        torch.testing.assert_close(got.cpu(), want, rtol=1e-7, atol=0)
