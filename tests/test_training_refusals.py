"""What the trainers' C entries refuse, on the host: every one of these calls returns before anything is launched, so no GPU is needed
and the addresses are never read."""

import ctypes
import math
from ctypes import byref, c_int64, c_void_p

import pytest

P, Q = 1 << 20, 1 << 30          # addresses that are only looked at


@pytest.fixture(scope="module")
def lib():
    import paper_1802_04819_b200 as slaq
    slaq.build()
    return slaq.load_library()


@pytest.mark.parametrize("change,code", [
    ({"type": 3}, -1), ({"type": -1}, -1), ({"rows": -1}, -1), ({"vocab": 0}, -1), ({"scale": 0.0}, -1), ({"scale": math.nan}, -1),
    ({"scale": math.inf}, -1), ({"scale": 2e30}, -1), ({"x": None}, -1), ({"stride": -4}, -1), ({"top": -1}, -1), ({"top": 3}, -1), ({"top": 33, "ids": P, "best": P}, -2),
    ({"vocab": (1 << 22) + 1}, -2), ({"rows": 1 << 31}, -2), ({"x": P + 2}, -1), ({"x": P + 1, "type": 1}, -1), ({"t": None}, -1),
    ({"rows": 0, "x": None, "t": None}, 0)])
def test_log_probabilities(lib, change, code):
    a = dict(x=P, type=0, rows=4, vocab=10, stride=10, t=P, scale=1.0, logprob=P, top=0, ids=None, best=None) | change
    assert lib.slaq_token_logprobs(a["x"], a["type"], a["rows"], a["vocab"], a["stride"], a["t"], a["scale"], a["logprob"], None, None, a["top"],
                                   a["ids"], a["best"], None) == code


@pytest.mark.parametrize("change,code", [
    ({"g": None}, -1), ({"t": None}, -1), ({"y": None}, -1), ({"norm": None}, -1), ({"h": P}, -1), ({"pitch": 9}, -1), ({"y": Q + 1}, -1),
    ({"y": P + 40}, -1), ({"y": P, "pitch": 12}, -1), ({"stride": 0, "y": P}, -1), ({"y": P + 40, "stride": 15, "pitch": 15}, -1),
    ({"y": P + 4}, -1), ({"scale": -2.0}, -1), ({"rows": 0, "x": None, "t": None, "g": None, "y": None, "norm": None}, 0)])
def test_gradients(lib, change, code):
    a = dict(x=P, rows=4, vocab=10, stride=10, t=Q, scale=1.0, norm=Q, e=None, g=Q, h=None, y=Q, pitch=10) | change
    assert lib.slaq_token_logprobs_grad(a["x"], 0, a["rows"], a["vocab"], a["stride"], a["t"], a["scale"], a["norm"], a["e"], a["g"], a["h"], a["y"],
                                        a["pitch"], None) == code
    if a["norm"] and not a["h"]:
        assert lib.slaq_token_loss(a["x"], 0, a["rows"], a["vocab"], a["stride"], a["t"], a["scale"], a["g"], None, a["y"], a["pitch"], None) == code


def test_job_losses(lib):
    assert lib.slaq_job_losses(-1, P, 5, None, P, None, P, None) == -1
    assert lib.slaq_job_losses(2, P, -5, None, P, None, P, None) == -1
    assert lib.slaq_job_losses(2, None, 5, None, P, None, P, None) == -1
    assert lib.slaq_job_losses(2, P, 5, None, None, None, P, None) == -1
    assert lib.slaq_job_losses(0, None, 0, None, None, None, None, None) == 0
    assert lib.slaq_job_row_grad(2, P, 5, None, None, None, 0, None) == -1
    assert lib.slaq_job_row_grad(0, None, 0, None, None, None, 0, None) == 0
    assert lib.slaq_job_row_grad(0, P, 5, None, None, P, 1, None) == -1
    assert lib.slaq_append_token_losses(None, 1, P, P, 5, None, P, None, None, None, P) == -1


@pytest.fixture
def plan():
    from paper_1802_04819_b200.training import _Tensor, _group

    def make(lib, tensors, groups=None, types=(0, 0), bits=32, ws=P, size=1 << 30, count=None):
        rows = (_Tensor * max(1, len(tensors)))()
        for row, t in zip(rows, tensors):
            for k, v in t.items():
                setattr(row, k, v)
        groups = [_group()] if groups is None else groups
        table = (type(_group()) * max(1, len(groups)))(*groups)
        h = c_void_p(5)
        rc = lib.slaq_adamw_create(ws, size, len(tensors) if count is None else count, rows, len(groups), table, types[0], types[1], bits, None, byref(h))
        assert rc < 0 and not h.value
        return rc
    return make


def _tensor(at=Q, n=100, **more):
    return dict(dict(param=at, grad=at + (1 << 24), exp_avg=at + (2 << 24), exp_avg_sq=at + (3 << 24), n=n, group=0), **more)


def test_plans(lib, plan):
    from paper_1802_04819_b200.training import _group
    far = _tensor(at=Q + (1 << 28))
    for tensors in ([_tensor(), _tensor()], [_tensor(), _tensor(at=Q + 396)], [_tensor(), far | dict(exp_avg=Q + 4)], [_tensor(n=-1)], [_tensor(group=1)],
                    [_tensor(group=-1)], [_tensor(param=None)], [_tensor(exp_avg=None)], [_tensor(exp_avg_sq=None)], [_tensor(grad=None)],
                    [_tensor(param=Q + 2)], [_tensor(grad=Q)], [_tensor(grad=Q + 399)], [_tensor(grad=Q - 396)], [_tensor(master=Q + 8)], [_tensor(), far | dict(master=8 << 28)]):
        assert plan(lib, tensors) == -1, tensors
    assert plan(lib, [_tensor()], bits=8) == -1                       # scales are missing
    assert plan(lib, [_tensor()], bits=16) == -1
    for types in ((3, 3), (0, 1), (1, 2), (2, 1), (0, -1)):
        assert plan(lib, [_tensor()], types=types) == -1
    for bad in (_group(lr=-1.0), _group(lr=math.nan), _group(betas=(1.0, 0.9)), _group(betas=(0.9, 1.0)), _group(eps=-1.0), _group(eps=math.inf),
                _group(weight_decay=math.inf), _group(grad_scale=math.nan), _group(step=-1)):
        assert plan(lib, [_tensor()], [bad]) == -1
    assert plan(lib, [_tensor()], []) == -1
    assert plan(lib, [_tensor()], count=-1) == -1
    assert plan(lib, [_tensor(n=(1 << 38) + 1)]) == -2


def test_sizes_of_a_plan(lib):
    sizes = (c_int64 * 3)(5, 0, 100_000)
    small = lib.slaq_adamw_workspace_bytes(3, ctypes.addressof(sizes), 2)
    sizes[1] = 50_000_000
    assert 0 < small < lib.slaq_adamw_workspace_bytes(3, ctypes.addressof(sizes), 2)
    sizes[1] = -1
    assert lib.slaq_adamw_workspace_bytes(3, ctypes.addressof(sizes), 2) == 0
    assert lib.slaq_adamw_workspace_bytes(3, ctypes.addressof(sizes), 0) == 0
    for call in (lib.slaq_adamw_step, lib.slaq_adamw_set_grads, lib.slaq_adamw_get_steps):
        assert call(None, None, None) == -1
    assert lib.slaq_adamw_destroy(None) == 0
