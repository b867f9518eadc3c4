"""Calls that a capture refuses leave the capture as it was."""

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_a_capture_goes_on_after_a_refused_call():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_1802_04819_b200 as slaq
    slaq.build()
    p, g, q, other = (torch.full((300,), x, device="cuda") for x in (1.0, 1.0, 1.0, 2.0))
    plan = slaq.AdamW([p], [g], groups=[dict(lr=0.1, weight_decay=0.0)])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        for call in (plan.get_steps, lambda: plan.set_grads([other]), lambda: slaq.AdamW([q], [g])):
            with pytest.raises(slaq.SlaqError) as e:
                call()
            assert e.value.code == -1
        plan.step()
    for _ in range(3):
        graph.replay()
    assert plan.get_steps().tolist() == [3]
    torch.testing.assert_close(p, torch.full_like(p, 0.7), rtol=0, atol=1e-5)
    plan.step()
    assert plan.get_steps().tolist() == [4]
