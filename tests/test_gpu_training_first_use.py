"""Kernels of the trainers' operators that are first used while a graph is being captured, in a process of their own: kernels are
loaded once per process."""

import subprocess
import sys
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu

ROOT = Path(__file__).resolve().parent.parent

CAPTURE = """
import sys
sys.path.insert(0, sys.argv[1])
import torch
import paper_1802_04819_b200 as slaq
x = torch.randn(6, int(sys.argv[2]), device="cuda").bfloat16()
t, g = torch.arange(6, device="cuda"), torch.full((6,), -0.5, device="cuda")
off = torch.tensor([0, 2, 6], device="cuda")
p = torch.ones(1000, device="cuda")
plan = slaq.AdamW([p], [torch.ones(1000, device="cuda")], groups=[dict(lr=0.1, weight_decay=0.0)], state_bits=8)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    a = slaq.token_logprobs(x, t, top=3)
    b = slaq.token_logprobs_grad(x, t, a.norm, g, entropy=a.entropy, grad_entropy=g)
    c = slaq.token_loss(x, t, g)
    d = slaq.job_losses(off, t, a.logprob), slaq.job_row_grad(off, t)
    plan.step()
for _ in range(2):
    graph.replay()
e = slaq.token_logprobs(x, t, top=3)
for u, v in ((a.logprob, e.logprob), (a.top_ids, e.top_ids), (b, slaq.token_logprobs_grad(x, t, e.norm, g, entropy=e.entropy, grad_entropy=g)),
             (c[1], slaq.token_loss(x, t, g)[1]), (d[0], slaq.job_losses(off, t, e.logprob)), (d[1], slaq.job_row_grad(off, t))):
    assert torch.equal(u, v)
torch.testing.assert_close(p, torch.full_like(p, 0.8), rtol=0, atol=1e-5)
assert plan.get_steps().tolist() == [2]
"""


@pytest.mark.parametrize("vocab", [10, 500, 3000, 150000])
def test_first_used_in_a_capture(vocab):
    import paper_1802_04819_b200 as slaq
    slaq.build()
    subprocess.run([sys.executable, "-c", CAPTURE, str(ROOT), str(vocab)], check=True, timeout=300)
