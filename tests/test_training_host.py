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
    sources = [CSRC / "slaq_adamw.cu", CSRC / "slaq_logprob.cu", CSRC / "slaq_job_loss.cu", ROOT / "tests" / "host_fakes" / "fake_training.cpp"]
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
    assert plan([_group(**numbers)])[0] == code
    _, h = plan()
    assert fake.slaq_adamw_set_group(h, 0, byref(_group(**{"step": -1, **numbers})), None) == code


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
