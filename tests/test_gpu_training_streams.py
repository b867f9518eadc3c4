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
