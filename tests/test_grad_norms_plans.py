"""Plans of gradients' norms on the host: nothing is launched, no GPU is needed, and the addresses are never read."""

import ctypes
import shutil
import subprocess
from ctypes import byref, c_int64, c_void_p
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent
CSRC = ROOT / "paper_1802_04819_b200" / "csrc"
A, B, C = 1 << 20, 1 << 21, 1 << 22          # addresses that are only looked at


@pytest.fixture(scope="module")
def lib():
    import paper_1802_04819_b200 as slaq
    slaq.build()
    return slaq.load_library()


@pytest.fixture(scope="module")
def fake(lib, tmp_path_factory):
    """The same code over a runtime that only pretends (host_fakes/fake_training.cpp)."""
    where = tmp_path_factory.mktemp("fake")
    inc = ["-I", str(ROOT / "include"), "-I", str(CSRC), "-I", str(Path(shutil.which("nvcc")).resolve().parent.parent / "include")]
    cuda = ["nvcc", "-gencode", "arch=compute_100a,code=compute_100a", "-cudart", "none", "-Xcompiler"]   # no machine code: none of it runs
    for tool, source in ((cuda, CSRC / "slaq_grad_norm.cu"), (["g++"], ROOT / "tests" / "host_fakes" / "fake_training.cpp")):
        subprocess.run([*tool, "-fPIC", "-O1", "-std=c++17", *inc, "-c", str(source), "-o", str(where / (source.stem + ".o"))], check=True)
    so = where / "libfake.so"
    subprocess.run(["g++", "-shared", "-Wl,-Bsymbolic", "-o", str(so), str(where / "slaq_grad_norm.o"), str(where / "fake_training.o")], check=True)
    made = ctypes.CDLL(str(so))
    for name in ("create", "destroy", "set_grads", "workspace_bytes"):
        name = "slaq_grad_norms_" + name
        getattr(made, name).argtypes, getattr(made, name).restype = getattr(lib, name).argtypes, getattr(lib, name).restype
    return made


def _tensors(*rows):
    from paper_1802_04819_b200.training import _GradTensor
    table = (_GradTensor * len(rows))()
    for t, (grad, out) in zip(table, rows):
        t.grad, t.out, t.n, t.group, t.type = grad, out, 100, 0, 0
    return table


def test_a_given_output_stays_where_it_is(fake):
    """Tensor 0 is written to A whatever its gradient, so no other gradient may come to lie there; tensor 1 is written in place, wherever that is."""
    h = c_void_p()
    assert fake.slaq_grad_norms_create(None, 0, 2, _tensors((A, A), (B, None)), 1, None, byref(h)) == 0
    rows = lambda *at: (c_void_p * 2)(*at)   # noqa: E731
    assert fake.slaq_grad_norms_set_grads(h, rows(C, A), None) == -1
    assert fake.slaq_grad_norms_set_grads(h, rows(C, B), None) == 0
    assert fake.slaq_grad_norms_set_grads(h, rows(A, C), None) == 0
    fake.slaq_grad_norms_destroy(h)


def test_how_many_groups_a_plan_may_have(lib):
    """2^30: the groups' numbers, and what a block's threads add to them, stay within 31 bits."""
    one = (c_int64 * 1)(10)
    assert lib.slaq_grad_norms_workspace_bytes(1, one, 1 << 30) > 1 << 34
    for groups in ((1 << 30) + 1, (1 << 31) - 300, (1 << 31) - 1):
        assert lib.slaq_grad_norms_workspace_bytes(1, one, groups) == 0
        h = c_void_p(1)
        assert lib.slaq_grad_norms_create(None, 0, 1, _tensors((A, None)), groups, None, byref(h)) == -2
        assert h.value is None
