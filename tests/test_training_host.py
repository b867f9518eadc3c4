"""Host code of the trainers' operators, built against a CUDA runtime that only pretends (host_fakes/fake_training.cpp): no GPU is
needed, nothing is launched, and what a test asks to fail fails."""

import ctypes
import shutil
import subprocess
from ctypes import byref, c_double, c_float, c_int, c_int32, c_int64, c_size_t, c_void_p
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent
CSRC = ROOT / "paper_1802_04819_b200" / "csrc"
P, Q = 1 << 20, 1 << 30          # addresses that are only looked at


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    where = tmp_path_factory.mktemp("fake")
    inc = ["-I", str(ROOT / "include"), "-I", str(CSRC), "-I", str(Path(shutil.which("nvcc")).resolve().parent.parent / "include")]
    sources = [CSRC / "slaq_adamw.cu", CSRC / "slaq_logprob.cu", CSRC / "slaq_job_loss.cu", *(ROOT / "tests" / "host_fakes" / name for name in ("fake_training.cpp", "fake_handle.cu"))]
    objects, running = [], []
    for source in sources:
        objects.append(str(where / (source.stem + ".o")))
        cuda = ["nvcc", "-gencode", "arch=compute_100a,code=sm_100a", "-cudart", "none", "-Xcompiler"]
        running.append(subprocess.Popen([*(cuda if source.suffix == ".cu" else ["g++"]), "-fPIC", "-O1", "-std=c++17", *inc, "-c", str(source), "-o", objects[-1]]))
    assert not any([p.wait() for p in running])
    so = where / "libfake.so"
    subprocess.run(["g++", "-shared", "-Wl,-Bsymbolic", "-o", str(so), *objects], check=True)
    lib = ctypes.CDLL(str(so))
    vp = c_void_p
    lib.slaq_token_loss.argtypes = [vp, c_int, c_int64, c_int32, c_int64, vp, c_float, vp, vp, vp, c_int64, vp]
    lib.slaq_adamw_create.argtypes = [vp, c_size_t, c_int32, vp, c_int32, vp, c_int, c_int, c_int, vp, vp]
    for name in ("step", "set_grads", "get_steps"):
        getattr(lib, "slaq_adamw_" + name).argtypes = [vp, vp, vp]
    lib.slaq_adamw_set_group.argtypes = [vp, c_int32, vp, vp]
    lib.slaq_adamw_destroy.argtypes = [vp]
    lib.fake_limit.argtypes = [vp]
    lib.fake_handle.restype = vp
    lib.fake_handle_end.argtypes = [vp]
    return lib


def _number(lib, name):
    return c_int.in_dll(lib, "fake_" + name)


@pytest.fixture
def plan(fake):
    from paper_1802_04819_b200.training import _group, _Tensor
    made = []

    def make(groups=None, n=100):
        table = (_Tensor * 1)()
        for k, v in dict(param=Q, grad=Q + (1 << 24), exp_avg=Q + (2 << 24), exp_avg_sq=Q + (3 << 24), n=n, group=0).items():
            setattr(table[0], k, v)
        groups = [_group()] if groups is None else groups
        h = c_void_p()
        rc = fake.slaq_adamw_create(None, 0, 1, table, len(groups), (type(_group()) * len(groups))(*groups), 0, 0, 32, None, byref(h))
        if rc == 0:
            made.append(h)
        return rc, h
    yield make
    for h in made:
        fake.slaq_adamw_destroy(h)


@pytest.mark.parametrize("eps,code", [(0.0, 0), (1e-8, 0), (2.0 ** -126, 0), (1.17e-38, -1), (1e-40, -1), (2.0 ** -149, -1), (1e-60, -1), (5e-324, -1)])
def test_an_epsilon_below_the_normal_numbers_is_refused(fake, plan, eps, code):
    """The kernel's reciprocal takes it for 0, and elements without gradients would get 0 x infinity."""
    from paper_1802_04819_b200.training import _group
    assert plan([_group(eps=eps)])[0] == code
    _, h = plan()
    assert fake.slaq_adamw_set_group(h, 0, byref(_group(eps=eps, step=-1)), None) == code


@pytest.mark.parametrize("numbers,code", [
    (dict(grad_scale=3e38), 0), (dict(grad_scale=-3e38), 0), (dict(grad_scale=1e39), -1), (dict(grad_scale=-1e300), -1), (dict(lr=1e20, weight_decay=1e18), 0),
    (dict(lr=1e20, weight_decay=1e20), -1), (dict(lr=1e25, betas=(1 - 1e-12, 0.9)), 0), (dict(lr=1e25, betas=(1 - 1e-15, 0.9)), -1), (dict(step=2 ** 53), 0),
    (dict(step=2 ** 53 + 1), -1), (dict(step=2 ** 63 - 1), -1)])
def test_numbers_that_a_step_in_32_bits_does_not_hold_are_refused(fake, plan, numbers, code):
    """An infinite factor makes NaN of elements that are 0; a count of 2^63 - 1 overflows with the next step."""
    from paper_1802_04819_b200.training import _group

    def group(step, numbers):
        g = _group(**{k: v for k, v in numbers.items() if k != "step"})
        g.step = numbers.get("step", step)
        return g
    assert plan([group(0, numbers)])[0] == code
    _, h = plan()
    assert fake.slaq_adamw_set_group(h, 0, byref(group(-1, numbers)), None) == code


def test_a_call_takes_no_shared_memory_from_another_threads(fake):
    """Rows of both sizes are kept by one kernel, in different amounts of shared memory.  What it may use belongs to the kernel, not to the
    call: a call between another thread's request and launch must not lower it."""
    def call(rows, vocab):
        assert fake.slaq_token_loss(P, 1, rows, vocab, vocab, Q, 1.0, Q, Q, 1 << 44, vocab, None) == 0
        return _last(fake)

    def _last(lib):
        return c_void_p.in_dll(lib, "fake_last_kernel").value, c_size_t.in_dll(lib, "fake_last_bytes").value
    calls = [call(*shape) for shape in ((4096, 147_000), (4096, 128_000), (2048, 50_001), (4096, 151_936))]
    assert len({kernel for kernel, _ in calls[:3]}) == 1 and len({size for _, size in calls}) == 4
    for kernel, size in calls:
        assert fake.fake_limit(kernel) >= size


ROWS = [("logprobs", dict(x=4, targets=8, logprob=4, entropy=4, norm=8, ids=4, best=4)),
        ("grad", dict(x=4, targets=8, norm=8, entropy=4, g=4, h=4, out=4)),
        ("loss", dict(x=4, targets=8, g=4, logprob=4, out=4)),
        ("row_grad", dict(offsets=8, targets=8, weights=4, out=4)),
        ("losses", dict(offsets=8, targets=8, logprob=4, weights=4, out=8)),
        ("append", dict(ids=4, offsets=8, targets=8, logprob=4, weights=4, times=8, cores=4, out=8))]


def _call(lib, kind, at, handle=None):
    """The call with these addresses."""
    vp = c_void_p
    a = {k: vp(v) for k, v in at.items()}
    rows = (a.get("x"), c_int(0), c_int64(4), c_int32(100), c_int64(100), a.get("targets"), c_float(1.0))
    if kind == "logprobs":
        return lib.slaq_token_logprobs(*rows, a["logprob"], a["entropy"], a["norm"], c_int32(3), a["ids"], a["best"], None)
    if kind == "grad":
        return lib.slaq_token_logprobs_grad(*rows, a["norm"], a["entropy"], a["g"], a["h"], a["out"], c_int64(100), None)
    if kind == "loss":
        return lib.slaq_token_loss(*rows, a["g"], a["logprob"], a["out"], c_int64(100), None)
    if kind == "row_grad":
        return lib.slaq_job_row_grad(c_int32(2), a["offsets"], c_int64(4), a["targets"], a["weights"], a["out"], c_int32(1), None)
    if kind == "losses":
        return lib.slaq_job_losses(c_int32(2), a["offsets"], c_int64(4), a["targets"], a["logprob"], a["weights"], a["out"], None)
    return lib.slaq_append_token_losses(vp(handle), c_int32(2), a["ids"], a["offsets"], c_int64(4), a["targets"], a["logprob"], a["weights"], a["times"], a["cores"], a["out"])


@pytest.mark.parametrize("kind,sizes", ROWS, ids=[k for k, _ in ROWS])
def test_addresses_that_their_elements_size_does_not_divide_are_refused(fake, kind, sizes):
    """The GPU would fault.  A refused call launches nothing, an append neither the losses."""
    handle = fake.fake_handle(c_int32(8)) if kind == "append" else None
    good = {k: (i + 1) << 32 for i, k in enumerate(sizes)}
    before = _number(fake, "launches").value
    assert _call(fake, kind, good, handle) == 0 and _number(fake, "launches").value == before + 1
    for name, size in sizes.items():
        for by in (1, size // 2):
            assert _call(fake, kind, {**good, name: good[name] + by}, handle) == -1, (name, by)
    assert _number(fake, "launches").value == before + 1
    if handle:
        fake.fake_handle_end(handle)


def test_a_list_of_groups_at_an_odd_address_is_refused(fake, plan):
    _, h = plan()
    assert fake.slaq_adamw_step(h, 1 << 32, None) == 0
    assert fake.slaq_adamw_step(h, (1 << 32) + 2, None) == -1


@pytest.mark.parametrize("failure", ["create", "set_grads", "set_grads copy", "get_steps"])
def test_an_error_does_not_become_that_of_a_later_step(fake, plan, failure):
    """The runtime keeps the error of a call that failed until it is asked for; a step that was launched is not to find it."""
    _, h = plan()
    grads = (c_void_p * 1)(Q + (9 << 24))
    if failure == "create":
        _number(fake, "copies_fail").value = 1
        assert plan()[0] == -5
    elif failure == "set_grads":
        _number(fake, "capture_query_fails").value = 1
        assert fake.slaq_adamw_set_grads(h, grads, None) == -1
    elif failure == "set_grads copy":
        _number(fake, "copies_fail").value = 1
        assert fake.slaq_adamw_set_grads(h, grads, None) == -5
    else:
        _number(fake, "copies_fail").value = 1
        assert fake.slaq_adamw_get_steps(h, (c_int64 * 1)(), None) == -5
    before = _number(fake, "launches").value
    assert fake.slaq_adamw_step(h, None, None) == 0 and _number(fake, "launches").value == before + 1
    assert fake.cudaGetLastError() == 0


def test_a_launch_that_fails_is_an_error_once(fake, plan):
    from paper_1802_04819_b200.training import _group
    _, h = plan()
    for call in (lambda: fake.slaq_adamw_step(h, None, None), lambda: fake.slaq_adamw_set_group(h, 0, byref(_group()), None), lambda: plan()[0]):
        _number(fake, "launches_fail").value = 1
        assert call() == -5 and _number(fake, "launches_fail").value == 0
        assert fake.cudaGetLastError() == 0
        assert call() == 0


def test_calls_that_wait_are_refused_while_the_stream_is_captured(fake, plan):
    """Waiting would end the capture with an error of its own."""
    _, h = plan()
    launches, copies = _number(fake, "launches").value, _number(fake, "copies").value
    _number(fake, "capturing").value = 1
    try:
        assert plan()[0] == -1
        assert fake.slaq_adamw_get_steps(h, (c_int64 * 1)(), None) == -1
        assert fake.slaq_adamw_set_grads(h, (c_void_p * 1)(Q + (9 << 24)), None) == -1
        assert _number(fake, "launches").value == launches and _number(fake, "copies").value == copies
        assert fake.slaq_adamw_step(h, None, None) == 0
    finally:
        _number(fake, "capturing").value = 0
    assert plan()[0] == 0
