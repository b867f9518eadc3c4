/*
 * Argument marshalling for Python: the two calls of a scheduler's loop (slaq_append_losses, slaq_schedule), and the calls of a
 * trainer's (at the end of the file).
 *
 * Through ctypes the pointers of four arrays cost about ten microseconds per append, more than the call's own work on the
 * host for a cluster of a few hundred jobs.  Here the arrays are taken through the buffer protocol; an argument
 * that is not a contiguous array of the right type makes the function return None, and the caller converts it.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

typedef int (*append_fn)(void*, int32_t, const int32_t*, const double*, const double*);
typedef int (*append_ex_fn)(void*, int32_t, const int32_t*, const double*, const double*, const int32_t*);
typedef int (*schedule_fn)(void*, double, int64_t, int32_t*);

/* 1: `v` holds a contiguous array of `size`-byte entries of kind `kind` ('i' or 'd'); 0: it does not (no error is set) */
static int take(PyObject* o, int flags, Py_ssize_t size, char kind, Py_buffer* v) {
    if (PyObject_GetBuffer(o, v, flags | PyBUF_C_CONTIGUOUS | PyBUF_FORMAT) != 0) {
        PyErr_Clear();
        return 0;
    }
    const char* f = v->format ? v->format : "B";
    const int match = f[0] == kind || (kind == 'i' && f[0] == 'l');
    if (v->itemsize != size || !match || f[1] != 0) {
        PyBuffer_Release(v);
        return 0;
    }
    return 1;
}

/* append(append address, append_ex address, handle, ids, losses, times or None, cores or None) -> status or None */
static PyObject* append(PyObject* self, PyObject* const* args, Py_ssize_t n_args) {
    (void)self;
    if (n_args != 7) {
        PyErr_SetString(PyExc_TypeError, "append takes 7 arguments");
        return NULL;
    }
    void* const plain = PyLong_AsVoidPtr(args[0]);
    void* const ex = PyLong_AsVoidPtr(args[1]);
    void* const handle = PyLong_AsVoidPtr(args[2]);
    if (PyErr_Occurred()) return NULL;
    Py_buffer v[4];
    int held = 0, fits = 1, rc = 0;
    const int has_times = args[5] != Py_None, has_cores = args[6] != Py_None;
    fits = take(args[3], PyBUF_SIMPLE, 4, 'i', &v[0]);
    held = fits;
    if (fits && (fits = take(args[4], PyBUF_SIMPLE, 8, 'd', &v[1]))) held = 2;
    if (fits && has_times && (fits = take(args[5], PyBUF_SIMPLE, 8, 'd', &v[2]))) held = 3;
    if (fits && has_cores && !has_times) fits = 0;
    if (fits && has_cores && (fits = take(args[6], PyBUF_SIMPLE, 4, 'i', &v[3]))) held = 4;
    const Py_ssize_t n = fits ? v[0].len / 4 : 0;
    if (fits && (v[1].len != 8 * n || (has_times && v[2].len != 8 * n) || (has_cores && v[3].len != 4 * n) || n > INT32_MAX))
        fits = 0;
    if (fits) {
        const double* const times = has_times ? (const double*)v[2].buf : NULL;
        Py_BEGIN_ALLOW_THREADS;
        if (has_cores)
            rc = ((append_ex_fn)ex)(handle, (int32_t)n, (const int32_t*)v[0].buf, (const double*)v[1].buf, times,
                                    (const int32_t*)v[3].buf);
        else
            rc = ((append_fn)plain)(handle, (int32_t)n, (const int32_t*)v[0].buf, (const double*)v[1].buf, times);
        Py_END_ALLOW_THREADS;
    }
    for (int i = 0; i < held; ++i) PyBuffer_Release(&v[i]);
    if (!fits) Py_RETURN_NONE;
    return PyLong_FromLong(rc);
}

/* schedule(address, handle, epoch seconds, cores, out array, entries it must have) -> status or None */
static PyObject* schedule(PyObject* self, PyObject* const* args, Py_ssize_t n_args) {
    (void)self;
    if (n_args != 6) {
        PyErr_SetString(PyExc_TypeError, "schedule takes 6 arguments");
        return NULL;
    }
    void* const fn = PyLong_AsVoidPtr(args[0]);
    void* const handle = PyLong_AsVoidPtr(args[1]);
    const double seconds = PyFloat_AsDouble(args[2]);
    const long long cores = PyLong_AsLongLong(args[3]);
    const Py_ssize_t want = PyLong_AsSsize_t(args[5]);
    if (PyErr_Occurred()) return NULL;
    Py_buffer v;
    if (!take(args[4], PyBUF_WRITABLE, 4, 'i', &v)) Py_RETURN_NONE;
    if (v.len < 4 * want) {
        PyBuffer_Release(&v);
        Py_RETURN_NONE;
    }
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = ((schedule_fn)fn)(handle, seconds, (int64_t)cores, (int32_t*)v.buf);
    Py_END_ALLOW_THREADS;
    PyBuffer_Release(&v);
    return PyLong_FromLong(rc);
}

/*
 * The trainers' calls.  Their arguments are addresses and numbers that Python has taken from tensors; through ctypes fourteen of them
 * cost two microseconds, of the nine that a small call takes.
 */
static PyObject *s_dtype, *s_get_device, *s_numel, *s_is_contiguous, *s_data_ptr;

/* 1: t.name() == want; 0: it is not; -1: an exception */
static int number_is(PyObject* t, PyObject* name, long long want) {
    PyObject* const v = PyObject_CallMethodNoArgs(t, name);
    if (!v) return -1;
    const long long n = PyLong_AsLongLong(v);
    Py_DECREF(v);
    return n == -1 && PyErr_Occurred() ? -1 : n == want;
}

/* address(tensor or None, dtype, entries, GPU) -> its address, None for None, False if it is not such a contiguous tensor */
static PyObject* address(PyObject* self, PyObject* const* args, Py_ssize_t n_args) {
    (void)self;
    if (n_args != 4) {
        PyErr_SetString(PyExc_TypeError, "address takes 4 arguments");
        return NULL;
    }
    PyObject* const t = args[0];
    if (t == Py_None) Py_RETURN_NONE;
    PyObject* const dtype = PyObject_GetAttr(t, s_dtype);
    if (!dtype) return NULL;
    Py_DECREF(dtype);
    int ok = dtype == args[1];
    if (ok) ok = number_is(t, s_get_device, PyLong_AsLongLong(args[3]));
    if (ok > 0) ok = number_is(t, s_numel, PyLong_AsLongLong(args[2]));
    if (ok > 0) ok = number_is(t, s_is_contiguous, 1);
    if (ok < 0 || PyErr_Occurred()) return NULL;
    if (!ok) Py_RETURN_FALSE;
    return PyObject_CallMethodNoArgs(t, s_data_ptr);
}

/* An address (None: null), or a whole number; errors are left to PyErr_Occurred(). */
static void* pointer_of(PyObject* o) { return o == Py_None ? NULL : PyLong_AsVoidPtr(o); }
static long long number_of(PyObject* o) { return PyLong_AsLongLong(o); }

typedef int (*logprobs_fn)(const void*, int, int64_t, int32_t, int64_t, const int64_t*, float, float*, float*, float*, int32_t, int32_t*, float*, void*);
typedef int (*grad_fn)(const void*, int, int64_t, int32_t, int64_t, const int64_t*, float, const float*, const float*, const float*, const float*, void*,
                       int64_t, void*);
typedef int (*loss_fn)(const void*, int, int64_t, int32_t, int64_t, const int64_t*, float, const float*, float*, void*, int64_t, void*);
typedef int (*sample_fn)(const void*, int, int64_t, int32_t, int64_t, const float*, double, const float*, int32_t, const int32_t*, double, const float*, double,
                         const float*, int64_t*, float*, float*, int32_t*, void*);
typedef int (*row_grad_fn)(int32_t, const int64_t*, int64_t, const int64_t*, const float*, float*, int32_t, void*);
typedef int (*losses_fn)(int32_t, const int64_t*, int64_t, const int64_t*, const float*, const float*, double*, void*);
typedef int (*step_fn)(void*, const int32_t*, void*);
typedef int (*step_factors_fn)(void*, const int32_t*, const float*, int32_t, const int32_t*, void*);
typedef int (*measure_fn)(void*, const int32_t*, double, double, const float*, float*, float*, void*);
typedef int (*apply_fn)(void*, const int32_t*, const float*, void*);

/* The first argument of each is the C function's address, the others are its own. */
#define CALL(name, count, type, ...)                                                     \
    static PyObject* name(PyObject* self, PyObject* const* a, Py_ssize_t n) {             \
        (void)self;                                                                      \
        if (n != (count)) {                                                              \
            PyErr_SetString(PyExc_TypeError, #name " takes another number of arguments"); \
            return NULL;                                                                 \
        }                                                                                \
        const type fn = (type)pointer_of(a[0]);                                          \
        __VA_ARGS__                                                                      \
    }
#define RUN(call)                      \
    if (PyErr_Occurred()) return NULL; \
    int rc;                            \
    Py_BEGIN_ALLOW_THREADS;            \
    rc = call;                         \
    Py_END_ALLOW_THREADS;              \
    return PyLong_FromLong(rc);

/* what the three calls on rows of logits begin with */
typedef struct {
    const void* x;
    int type;
    int64_t rows, pitch;
    int32_t vocab;
    const int64_t* targets;
    float scale;
} Logits;
static Logits logits_of(PyObject* const* a) {
    Logits l;
    l.x = pointer_of(a[1]);
    l.type = (int)number_of(a[2]);
    l.rows = number_of(a[3]);
    const long long vocab = number_of(a[4]);
    l.vocab = vocab > INT32_MAX ? INT32_MAX : (int32_t)vocab;
    l.pitch = number_of(a[5]);
    l.targets = pointer_of(a[6]);
    l.scale = (float)PyFloat_AsDouble(a[7]);
    return l;
}

CALL(token_logprobs, 15, logprobs_fn, {
    const Logits l = logits_of(a);
    float *const logprob = pointer_of(a[8]), *const entropy = pointer_of(a[9]), *const norm = pointer_of(a[10]);
    const int32_t top = (int32_t)number_of(a[11]);
    int32_t* const ids = pointer_of(a[12]);
    float* const best = pointer_of(a[13]);
    void* const stream = pointer_of(a[14]);
    RUN(fn(l.x, l.type, l.rows, l.vocab, l.pitch, l.targets, l.scale, logprob, entropy, norm, top, ids, best, stream))
})
CALL(token_logprobs_grad, 15, grad_fn, {
    const Logits l = logits_of(a);
    const float *const norm = pointer_of(a[8]), *const entropy = pointer_of(a[9]), *const g = pointer_of(a[10]), *const h = pointer_of(a[11]);
    void* const out = pointer_of(a[12]);
    const int64_t pitch = number_of(a[13]);
    void* const stream = pointer_of(a[14]);
    RUN(fn(l.x, l.type, l.rows, l.vocab, l.pitch, l.targets, l.scale, norm, entropy, g, h, out, pitch, stream))
})
CALL(token_loss, 13, loss_fn, {
    const Logits l = logits_of(a);
    const float* const g = pointer_of(a[8]);
    float* const logprob = pointer_of(a[9]);
    void* const out = pointer_of(a[10]);
    const int64_t pitch = number_of(a[11]);
    void* const stream = pointer_of(a[12]);
    RUN(fn(l.x, l.type, l.rows, l.vocab, l.pitch, l.targets, l.scale, g, logprob, out, pitch, stream))
})
CALL(sample_tokens, 20, sample_fn, {
    const void* const x = pointer_of(a[1]);
    const int type = (int)number_of(a[2]);
    const int64_t rows = number_of(a[3]);
    const long long vocab = number_of(a[4]);
    const int64_t pitch = number_of(a[5]);
    const float* const uniform = pointer_of(a[6]);
    const double temperature = PyFloat_AsDouble(a[7]);
    const float* const temperatures = pointer_of(a[8]);
    const long long k = number_of(a[9]);
    const int32_t* const ks = pointer_of(a[10]);
    const double p = PyFloat_AsDouble(a[11]);
    const float* const ps = pointer_of(a[12]);
    const double q = PyFloat_AsDouble(a[13]);
    const float* const qs = pointer_of(a[14]);
    int64_t* const token = pointer_of(a[15]);
    float *const logprob = pointer_of(a[16]), *const kept_logprob = pointer_of(a[17]);
    int32_t* const kept = pointer_of(a[18]);
    void* const stream = pointer_of(a[19]);
    RUN(fn(x, type, rows, vocab > INT32_MAX ? INT32_MAX : (int32_t)vocab, pitch, uniform, temperature, temperatures,
           k > INT32_MAX ? INT32_MAX : k < 0 ? 0 : (int32_t)k, ks, p, ps, q, qs, token, logprob, kept_logprob, kept, stream))
})
CALL(job_row_grad, 9, row_grad_fn, {
    const long long jobs = number_of(a[1]);
    const int64_t *const offsets = pointer_of(a[2]), rows = number_of(a[3]), *const targets = pointer_of(a[4]);
    const float* const weights = pointer_of(a[5]);
    float* const out = pointer_of(a[6]);
    const int32_t zero_rest = (int32_t)number_of(a[7]);
    void* const stream = pointer_of(a[8]);
    RUN(jobs > INT32_MAX ? -2 : fn((int32_t)jobs, offsets, rows, targets, weights, out, zero_rest, stream))
})
CALL(job_losses, 9, losses_fn, {
    const long long jobs = number_of(a[1]);
    const int64_t *const offsets = pointer_of(a[2]), rows = number_of(a[3]), *const targets = pointer_of(a[4]);
    const float *const logprob = pointer_of(a[5]), *const weights = pointer_of(a[6]);
    double* const out = pointer_of(a[7]);
    void* const stream = pointer_of(a[8]);
    RUN(jobs > INT32_MAX ? -2 : fn((int32_t)jobs, offsets, rows, targets, logprob, weights, out, stream))
})
CALL(adamw_step, 4, step_fn, {
    void* const plan = pointer_of(a[1]);
    const int32_t* const active = pointer_of(a[2]);
    void* const stream = pointer_of(a[3]);
    RUN(fn(plan, active, stream))
})
CALL(adamw_step_factors, 7, step_factors_fn, {
    void* const plan = pointer_of(a[1]);
    const int32_t* const active = pointer_of(a[2]);
    const float* const factors = pointer_of(a[3]);
    const long long n_factors = number_of(a[4]);
    const int32_t* const factor_of = pointer_of(a[5]);
    void* const stream = pointer_of(a[6]);
    RUN(n_factors > INT32_MAX ? -2 : fn(plan, active, factors, (int32_t)n_factors, factor_of, stream))
})
CALL(grad_norms_measure, 9, measure_fn, {
    void* const plan = pointer_of(a[1]);
    const int32_t* const active = pointer_of(a[2]);
    const double scale = PyFloat_AsDouble(a[3]), most = PyFloat_AsDouble(a[4]);
    const float* const mosts = pointer_of(a[5]);
    float *const norm = pointer_of(a[6]), *const factor = pointer_of(a[7]);
    void* const stream = pointer_of(a[8]);
    RUN(fn(plan, active, scale, most, mosts, norm, factor, stream))
})
CALL(grad_norms_apply, 5, apply_fn, {
    void* const plan = pointer_of(a[1]);
    const int32_t* const active = pointer_of(a[2]);
    const float* const factor = pointer_of(a[3]);
    void* const stream = pointer_of(a[4]);
    RUN(fn(plan, active, factor, stream))
})

#define METHOD(name, text) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, text}
static PyMethodDef methods[] = {
    {"append", (PyCFunction)(void (*)(void))append, METH_FASTCALL, "one slaq_append_losses / slaq_append_losses_ex call"},
    {"schedule", (PyCFunction)(void (*)(void))schedule, METH_FASTCALL, "one slaq_schedule call"},
    METHOD(address, "the address of a contiguous tensor of a type and size on a GPU"),
    METHOD(token_logprobs, "one slaq_token_logprobs call"),
    METHOD(token_logprobs_grad, "one slaq_token_logprobs_grad call"),
    METHOD(token_loss, "one slaq_token_loss call"),
    METHOD(sample_tokens, "one slaq_sample_tokens call"),
    METHOD(job_row_grad, "one slaq_job_row_grad call"),
    METHOD(job_losses, "one slaq_job_losses call"),
    METHOD(adamw_step, "one slaq_adamw_step call"),
    METHOD(adamw_step_factors, "one slaq_adamw_step_factors call"),
    METHOD(grad_norms_measure, "one slaq_grad_norms_measure call"),
    METHOD(grad_norms_apply, "one slaq_grad_norms_apply call"),
    {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__marshal(void) {
    s_dtype = PyUnicode_InternFromString("dtype");
    s_get_device = PyUnicode_InternFromString("get_device");
    s_numel = PyUnicode_InternFromString("numel");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    if (!s_dtype || !s_get_device || !s_numel || !s_is_contiguous || !s_data_ptr) return NULL;
    return PyModule_Create(&module);
}
