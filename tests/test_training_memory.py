"""Whose memory the trainers' calls take, with objects that only look like torch's: no GPU is needed, nothing is launched."""

import contextlib
from types import SimpleNamespace

import pytest


class Tensor:
    """What the calls ask of a tensor.  `stream` is the one that was current when it was made."""

    def __init__(self, dtype, n, stream):
        self.dtype, self.n, self.stream, self.recorded, self.is_cuda, self.requires_grad = dtype, n, stream, [], True, False
        self.device = SimpleNamespace(index=0)

    def to(self, dtype):
        return Tensor(dtype, self.n, self.stream)

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
    fake = SimpleNamespace(cuda=cuda, empty=make, zeros=make, **{t: getattr(torch, t) for t in ("int64", "int32", "float32", "float64", "uint8", "float8_e4m3fn")})
    monkeypatch.setattr(training, "_torch", fake)
    monkeypatch.setattr(training, "_current_stream", lambda gpu: w.stream)
    monkeypatch.setattr(training, "_current_device", lambda: 0)
    monkeypatch.setattr(training, "_changed", lambda t: None)
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


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("call", ["step", "set_group", "set_grads", "get_steps"])
def test_a_plans_memory_is_kept_for_every_stream_that_uses_it(world, monkeypatch, bits, call):
    """Dropped after a call on another stream, it must not go back to the one it was made on before the other has passed the call: its
    tables, and the states that it made."""
    t = world.torch
    lib = SimpleNamespace(**{"slaq_adamw_" + name: lambda *a: 0 for name in ("create", "destroy", "set_group", "set_grads", "get_steps")},
                          slaq_adamw_workspace_bytes=lambda *a: 4096)
    monkeypatch.setattr(world.training, "load_library", lambda: lib)
    monkeypatch.setattr(world.training, "_calls", SimpleNamespace(adamw_step=lambda *a: 0))
    weights, grads = [Tensor(t.float32, n, 5) for n in (300, 7)], [Tensor(t.float32, n, 5) for n in (300, 7)]
    plan = world.slaq.AdamW(weights, grads, state_bits=bits)
    own = [plan._ws, *plan.exp_avg, *plan.exp_avg_sq, *(plan.exp_avg_scale or []), *(plan.exp_avg_sq_scale or [])]
    assert len(own) == (9 if bits == 8 else 5)

    def use(stream):
        {"step": plan.step, "set_group": lambda stream: plan.set_group(0, stream=stream, lr=0.1), "set_grads": lambda stream: plan.set_grads(grads, stream=stream),
         "get_steps": plan.get_steps}[call](stream=stream)
    use(None)
    assert not any(x.recorded for x in own)                  # the stream that it was made on
    for _ in range(2):
        use(9)
        use(0)
    assert all(x.recorded == [9, 0] for x in own)            # once for each
    assert not any(x.recorded for x in weights + grads)      # the caller's


def test_a_stream_of_another_gpu_is_refused(world):
    """Its calls would run on the current stream of the tensors' GPU, which is ordered behind nothing of that stream's."""
    t = world.torch
    there = SimpleNamespace(device=SimpleNamespace(index=1), cuda_stream=9)
    offsets, targets = Tensor(t.int64, 4, 5), Tensor(t.int64, 20, 5)
    with pytest.raises(world.slaq.SlaqError, match="another GPU"):
        world.slaq.job_row_grad(offsets, targets, stream=there)
    assert not world.made


def test_rows_on_another_gpu_than_the_schedulers_are_refused(world, monkeypatch):
    t = world.torch
    monkeypatch.setattr(Tensor, "get_device", lambda self: 1)
    sched = SimpleNamespace(_stream=5, _h=None, _check=lambda rc: rc, _lib=SimpleNamespace(slaq_append_token_losses=lambda *a: pytest.fail("called")))
    args = [Tensor(t.int32, 3, 5), Tensor(t.int64, 4, 5), Tensor(t.int64, 20, 5), Tensor(t.float32, 20, 5)]
    with pytest.raises(world.slaq.SlaqError, match="another GPU"):
        world.training.append_token_losses(sched, *args, None, None, None, None)


@pytest.mark.parametrize("changes", [dict(group_of=[0, 2 ** 32]), dict(group_of=[-(2 ** 32), 0]), dict(group_of=[0, 1]), dict(groups=[dict(step=2 ** 64)]),
                                     dict(groups=[dict(step=2 ** 53 + 1)]), dict(groups=[dict(step=-1)])])
def test_numbers_that_their_fields_do_not_hold_are_refused(world, monkeypatch, changes):
    """2^32 is 0 in 32 bits: the tensor would have been stepped with group 0."""
    t = world.torch
    lib = SimpleNamespace(slaq_adamw_create=lambda *a: 0, slaq_adamw_destroy=lambda *a: 0, slaq_adamw_set_group=lambda *a: 0, slaq_adamw_workspace_bytes=lambda *a: 4096)
    monkeypatch.setattr(world.training, "load_library", lambda: lib)
    weights, grads = [Tensor(t.float32, n, 5) for n in (300, 7)], [Tensor(t.float32, n, 5) for n in (300, 7)]
    with pytest.raises(world.slaq.SlaqError) as e:
        world.slaq.AdamW(weights, grads, **changes)
    assert e.value.code == -1
    plan = world.slaq.AdamW(weights, grads)
    with pytest.raises(world.slaq.SlaqError):
        plan.set_group(0, step=2 ** 64)
    plan.set_group(0, lr=0.1)
