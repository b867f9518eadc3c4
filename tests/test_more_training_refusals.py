"""What sampling, the gradients' norms and the step with factors refuse, on the host: nothing is launched, no GPU is needed, and the addresses are
never read.  Host code where the runtime fails is built against one that only pretends (host_fakes/fake_training.cpp)."""

import ctypes
import math
import shutil
import subprocess
from ctypes import byref, c_int, c_int64, c_void_p
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent
CSRC = ROOT / "paper_1802_04819_b200" / "csrc"
P, Q = 1 << 20, 1 << 30          # addresses that are only looked at


@pytest.fixture(scope="module")
def lib():
    import paper_1802_04819_b200 as slaq
    slaq.build()
    return slaq.load_library()


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    where = tmp_path_factory.mktemp("fake")
    (where / "more.cpp").write_text('extern "C" void __cudaRegisterVar(void**, char*, char*, const char*, int, unsigned long, int, int) {}\n')
    inc = ["-I", str(ROOT / "include"), "-I", str(CSRC), "-I", str(Path(shutil.which("nvcc")).resolve().parent.parent / "include")]
    sources = [CSRC / "slaq_adamw.cu", CSRC / "slaq_grad_norm.cu", CSRC / "slaq_sample.cu", ROOT / "tests" / "host_fakes" / "fake_training.cpp", where / "more.cpp"]
    objects, running = [], []
    for source in sources:
        objects.append(str(where / (source.stem + ".o")))
        cuda = ["nvcc", "-gencode", "arch=compute_100a,code=compute_100a", "-cudart", "none", "-Xcompiler"]   # no machine code: none of it runs
        running.append(subprocess.Popen([*(cuda if source.suffix == ".cu" else ["g++"]), "-fPIC", "-O1", "-std=c++17", *inc, "-c", str(source), "-o", objects[-1]]))
    assert not any([p.wait() for p in running])
    so = where / "libfake.so"
    subprocess.run(["g++", "-shared", "-Wl,-Bsymbolic", "-o", str(so), *objects], check=True)
    lib = ctypes.CDLL(str(so))
    import paper_1802_04819_b200.binding as binding
    real = binding.load_library()
    for name in binding.EXPORTED_SYMBOLS:
        if name.startswith(("slaq_adamw", "slaq_grad_norms", "slaq_sample")):
            getattr(lib, name).argtypes, getattr(lib, name).restype = getattr(real, name).argtypes, getattr(real, name).restype
    return lib


def _number(lib, name):
    return c_int.in_dll(lib, "fake_" + name)


def _sample(lib, change):
    a = dict(x=P, type=0, rows=4, vocab=10, stride=10, u=P, T=1.0, Ts=None, k=0, ks=None, p=1.0, ps=None, q=0.0, qs=None, token=Q, logprob=Q, kept_logprob=Q, kept=Q) | change
    return lib.slaq_sample_tokens(a["x"], a["type"], a["rows"], a["vocab"], a["stride"], a["u"], a["T"], a["Ts"], a["k"], a["ks"], a["p"], a["ps"], a["q"], a["qs"],
                                  a["token"], a["logprob"], a["kept_logprob"], a["kept"], None)


BAD = [({"type": 3}, -1), ({"rows": -1}, -1), ({"vocab": 0}, -1), ({"vocab": (1 << 22) + 1}, -2), ({"rows": 1 << 31}, -2), ({"x": None}, -1), ({"u": None}, -1),
       ({"token": None}, -1), ({"stride": -1}, -1), ({"x": P + 2}, -1), ({"x": P + 1, "type": 1}, -1), ({"u": P + 2}, -1), ({"Ts": P + 1}, -1), ({"ks": P + 2}, -1),
       ({"ps": P + 3}, -1), ({"qs": P + 2}, -1), ({"token": Q + 4}, -1), ({"logprob": Q + 2}, -1), ({"kept_logprob": Q + 2}, -1), ({"kept": Q + 2}, -1),
       ({"T": -1.0}, -1), ({"T": math.nan}, -1), ({"T": 1e-31}, -1), ({"T": 1e31}, -1), ({"T": math.inf}, -1), ({"p": 1.1}, -1), ({"p": -0.1}, -1), ({"p": math.nan}, -1),
       ({"q": 1.5}, -1), ({"q": -1.0}, -1), ({"q": math.nan}, -1), ({"rows": 0, "x": None, "u": None, "token": None}, 0)]


@pytest.mark.parametrize("change,code", BAD)
def test_samples(lib, fake, change, code):
    assert _sample(lib, change) == code
    before = _number(fake, "launches").value
    assert _sample(fake, change) == code and _number(fake, "launches").value == before


@pytest.mark.parametrize("change", [{}, {"k": 5}, {"kept": None}, {"T": 0.0}, {"T": -1.0, "Ts": P}, {"p": 7.0, "ps": P}, {"q": 7.0, "qs": P}, {"k": -3},
                                    {"vocab": 10_000, "stride": 10_000, "rows": 1000}, {"vocab": 300, "stride": 300}, {"vocab": 200_000, "stride": 200_000, "type": 1}])
def test_a_sample_is_launched_and_an_error_of_a_launch_is_not_left_behind(fake, change):
    assert _sample(fake, change) == 0
    _number(fake, "launches_fail").value = 1
    assert _sample(fake, change) == -5
    assert _sample(fake, change) == 0


def _tensors(*rows):
    from paper_1802_04819_b200.training import _GradTensor
    table = (_GradTensor * len(rows))()
    for t, (grad, out, n, group, kind) in zip(table, rows):
        t.grad, t.out, t.n, t.group, t.type = grad, out, n, group, kind
    return table


@pytest.mark.parametrize("rows,groups,code", [
    ([(Q, None, 10, 1, 0)], 1, -1), ([(Q, None, 10, -1, 0)], 1, -1), ([(Q, None, 10, 0, 3)], 1, -1), ([(Q, None, -1, 0, 0)], 1, -1), ([(None, None, 10, 0, 0)], 1, -1),
    ([(Q + 2, None, 10, 0, 0)], 1, -1), ([(Q, Q + (1 << 20) + 1, 10, 0, 1)], 1, -1), ([(Q, None, 10, 0, 0), (Q, None, 10, 0, 0)], 1, -1),
    ([(Q, None, 10, 0, 0), (Q + 36, None, 10, 0, 0)], 1, -1), ([(Q, Q + 20, 10, 0, 0)], 1, -1), ([(Q, Q + 4096, 10, 0, 0), (Q + 4096, None, 3, 0, 0)], 1, -1),
    ([(Q, None, (1 << 38) + 1, 0, 0)], 1, -2), ([(Q, None, 10, 0, 0)], 0, -1)])
def test_plans_of_norms(lib, fake, rows, groups, code):
    for where in (lib, fake):
        h = c_void_p(1)
        assert where.slaq_grad_norms_create(None, 0, len(rows), _tensors(*rows), groups, None, byref(h)) == code
        assert h.value is None
    assert lib.slaq_grad_norms_create(None, 0, 1, None, 1, None, byref(h)) == -1 and lib.slaq_grad_norms_create(None, 0, 0, None, 1, None, None) == -1


def test_sizes_of_the_workspace(lib):
    def need(numels, groups):
        return lib.slaq_grad_norms_workspace_bytes(len(numels), (c_int64 * len(numels))(*numels), groups)
    assert need([10], 0) == 0 and need([-1], 1) == 0 and need([(1 << 38) + 1], 1) == 0 and need([1 << 38], 1) > 0 and need([1 << 37] * 3, 1) == 0
    assert 0 < need([10], 1) < need([10_000_000], 1)
    assert lib.slaq_grad_norms_destroy(None) == 0 and lib.slaq_grad_norms_last_error(None) == b"null handle"
    assert lib.slaq_grad_norms_measure(None, None, 1.0, 1.0, None, P, P, None) == -1 and lib.slaq_grad_norms_apply(None, None, P, None) == -1
    assert lib.slaq_grad_norms_set_grads(None, None, None) == -1 and lib.slaq_adamw_step_factors(None, None, None, 0, None, None) == -1


@pytest.fixture
def norms(fake):
    made = []

    def make(groups=2, expect=0):
        h = c_void_p()
        rc = fake.slaq_grad_norms_create(None, 0, 2, _tensors((Q, None, 100, 0, 0), (Q + 4096, Q + 8192, 100, groups - 1, 1)), groups, None, byref(h))
        assert rc == expect
        if rc == 0:
            made.append(h)
        return h
    yield make
    for h in made:
        fake.slaq_grad_norms_destroy(h)


def test_calls_of_a_plan(fake, norms):
    h = norms()
    before = _number(fake, "launches").value
    for bad in ((P + 2, 1.0, 1.0, None, P, P), (None, 1.0, 1.0, P + 1, P, P), (None, 1.0, 1.0, None, None, P), (None, 1.0, 1.0, None, P + 2, P), (None, 1.0, 1.0, None, P, P + 2),
                (None, 1.0, -1.0, None, P, P), (None, 1.0, math.nan, None, P, P), (None, math.inf, 1.0, None, P, P), (None, math.nan, 1.0, None, P, P), (None, 4e38, 1.0, None, P, P)):
        assert fake.slaq_grad_norms_measure(h, *bad, None) == -1
    for bad in ((P + 2, P), (None, None), (None, P + 1)):
        assert fake.slaq_grad_norms_apply(h, *bad, None) == -1
    assert _number(fake, "launches").value == before
    for good in ((P, -0.5, math.inf, None, P, None), (None, 1.0, 0.0, P, P, P)):
        assert fake.slaq_grad_norms_measure(h, *good, None) == 0
    assert fake.slaq_grad_norms_apply(h, P, P, None) == 0
    _number(fake, "launches_fail").value = 1
    assert fake.slaq_grad_norms_measure(h, None, 1.0, 1.0, None, P, P, None) == -5 and b"launched" in fake.slaq_grad_norms_last_error(h)
    assert fake.slaq_grad_norms_measure(h, None, 1.0, 1.0, None, P, P, None) == 0
    _number(fake, "launches_fail").value = 1
    assert fake.slaq_grad_norms_apply(h, None, P, None) == -5
    many = norms(groups=5000)
    before = _number(fake, "launches").value
    assert fake.slaq_grad_norms_measure(many, None, 1.0, 1.0, None, P, P, None) == 0 and _number(fake, "launches").value == before + 2


def test_other_gradients_and_captures(fake, norms):
    h = norms()
    rows = lambda *at: (c_void_p * 2)(*at)   # noqa: E731
    assert fake.slaq_grad_norms_set_grads(h, None, None) == -1
    for bad in (rows(None, Q), rows(Q + 2, Q + 4096), rows(Q + (1 << 20), Q + 8192 + 2), rows(Q + 8192, Q + 4096)):
        assert fake.slaq_grad_norms_set_grads(h, bad, None) == -1
    assert fake.slaq_grad_norms_set_grads(h, rows(Q + (1 << 20), Q + (2 << 20)), None) == 0
    _number(fake, "capturing").value = 1
    try:
        assert fake.slaq_grad_norms_set_grads(h, rows(Q, Q + 4096), None) == -1
        assert fake.slaq_grad_norms_measure(h, None, 1.0, 1.0, None, P, P, None) == 0       # the others are captured
        norms(expect=-1)
    finally:
        _number(fake, "capturing").value = 0
    _number(fake, "copies_fail").value = 1
    assert fake.slaq_grad_norms_set_grads(h, rows(Q, Q + 4096), None) == -5


def test_factors_of_a_step(fake):
    from paper_1802_04819_b200.training import _group, _Tensor
    table = (_Tensor * 1)()
    for k, v in dict(param=Q, grad=Q + (1 << 24), exp_avg=Q + (2 << 24), exp_avg_sq=Q + (3 << 24), n=100, group=0).items():
        setattr(table[0], k, v)
    h = c_void_p()
    assert fake.slaq_adamw_create(None, 0, 1, table, 2, (type(_group()) * 2)(_group(), _group()), 0, 0, 32, None, byref(h)) == 0
    for bad in ((None, P, 1, None), (None, P, 3, None), (None, P, 0, P), (None, P + 2, 2, None), (None, P, 2, P + 1), (None, None, 2, None), (None, None, 0, P), (P + 1, P, 2, None)):
        assert fake.slaq_adamw_step_factors(h, *bad, None) == -1
    for good in ((None, P, 2, None), (P, P, 7, P), (None, None, 0, None)):
        assert fake.slaq_adamw_step_factors(h, *good, None) == 0
    fake.slaq_adamw_destroy(h)


