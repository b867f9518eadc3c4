"""Whose memory the trainers' calls take, with objects that only look like torch's: no GPU is needed, nothing is launched."""

import contextlib
from types import SimpleNamespace

import pytest


class Tensor:
    """What the calls ask of a tensor.  `stream` is the one that was current when it was made."""

    def __init__(self, dtype, n, stream):
        self.dtype, self.n, self.stream, self.device, self.recorded = dtype, n, stream, "cuda:0", []

    def numel(self):
        return self.n

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20

    def record_stream(self, stream):
        self.recorded.append(stream)


@pytest.fixture
def world(monkeypatch):
    """A torch whose current stream is 5; `world.made` are the tensors that the calls allocate."""
    import torch

    import paper_1802_04819_b200 as slaq
    slaq.build()
    from paper_1802_04819_b200 import training
    training._load()
    w = SimpleNamespace(stream=5, made=[], training=training, slaq=slaq)

    @contextlib.contextmanager
    def current(stream):
        before, w.stream = w.stream, stream
        yield
        w.stream = before

    def make(*shape, dtype=torch.float32, device=None):
        n = 1
        for s in shape:
            n *= s
        w.made.append(Tensor(dtype, n, w.stream))
        return w.made[-1]
    cuda = SimpleNamespace(device=lambda d: contextlib.nullcontext(), stream=current, default_stream=lambda d: 0, ExternalStream=lambda raw, device: raw)
    fake = SimpleNamespace(cuda=cuda, empty=make, zeros=make, int64=torch.int64, int32=torch.int32, float32=torch.float32, float64=torch.float64)
    monkeypatch.setattr(training, "_torch", fake)
    monkeypatch.setattr(training, "_current_stream", lambda gpu: w.stream)
    monkeypatch.setattr(training, "_current_device", lambda: 0)
    w.torch = fake
    return w


@pytest.mark.parametrize("handle", [5, 9, 0])
def test_the_losses_that_an_append_makes_are_its_streams(world, handle):
    """Memory of the current stream may still be in use there, and is given away there while the handle's stream works on it."""
    t = world.torch
    calls = []
    sched = SimpleNamespace(_stream=handle, _h=None, _check=lambda rc: rc, _lib=SimpleNamespace(slaq_append_token_losses=lambda *a: calls.append(a) or 0))
    args = [Tensor(t.int32, 3, 5), Tensor(t.int64, 4, 5), Tensor(t.int64, 20, 5), Tensor(t.float32, 20, 5)]
    out = world.training.append_token_losses(sched, *args, None, None, None, None)
    assert calls and world.made == [out] and out.n == 3 and out.stream == handle
    given = Tensor(t.float64, 3, 5)
    assert world.training.append_token_losses(sched, *args, None, None, None, given) is given and len(world.made) == 1


def test_a_scheduler_knows_the_stream_it_was_given(world):
    sched = world.slaq.Scheduler.__new__(world.slaq.Scheduler)
    sched._h, rc = None, [0]
    sched._lib = SimpleNamespace(slaq_set_stream=lambda h, raw: rc[0], slaq_last_error=lambda h: b"no")
    for stream, raw in ((SimpleNamespace(cuda_stream=77), 77), (78, 78), (None, 0), (SimpleNamespace(cuda_stream=0), 0)):
        sched.set_stream(stream)
        assert sched._stream == raw
    rc[0] = -5
    with pytest.raises(world.slaq.SlaqError):
        sched.set_stream(99)
    assert sched._stream == 0
