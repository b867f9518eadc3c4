"""What a trainer computes beside the scheduler, on torch CUDA tensors: same names as the C ABI, argument marshalling only.

A training step of many jobs whose logits lie in one matrix, job j's rows being ``offsets[j] .. offsets[j + 1]``:

    row_grad = slaq.job_row_grad(offsets, targets)                    # derivative of each job's mean loss by its rows
    logprob, grad = slaq.token_loss(logits, targets, row_grad)        # log probabilities, gradient by the logits
    sched.append_token_losses(job_ids, offsets, targets, logprob)     # the jobs' losses, into their histories
    ...                                                               # the model's own backward pass
    adamw.step(active=alloc)                                          # only the jobs that were given cores

Every call is asynchronous on ``stream`` (a torch stream or a raw cudaStream_t; default: torch's current stream of the
tensors' device; ``append_token_losses`` is on the handle's).  Results that are not given as ``out`` are allocated by torch for
that stream; inputs must be ready on it, and stay alive until it has passed the call.  No call records anything for autograd:
logits that require a gradient are given it by ``logits.backward(grad)``.  A given ``out``, and weights that require a gradient,
count as changed in place (in a CUDA graph: when it is captured).  Refusals raise ``SlaqError``.
"""

from __future__ import annotations

import contextlib
import ctypes
from ctypes import c_double, c_int32, c_int64, c_void_p
from typing import NamedTuple

import numpy as np

from .binding import SlaqError, _marshal, load_library

F32, BF16, F16 = 0, 1, 2
MAX_VOCAB, MAX_TOP = 1 << 22, 32
STATE_BLOCK = 256

_torch = _calls = _address = _current_stream = _current_device = _changed = None
_types, _at = {}, {}          # element types; the addresses of the C functions


def _load():
    global _torch, _calls, _address, _current_stream, _current_device, _changed
    if _torch is None:
        import torch
        lib, _calls = load_library(), _marshal()
        for name in ("token_logprobs", "token_logprobs_grad", "token_loss", "job_row_grad", "job_losses", "adamw_step"):
            _at[name] = ctypes.cast(getattr(lib, "slaq_" + name), c_void_p).value
        _address = _calls.address
        _types.update({torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16})
        # the address alone: torch.cuda.current_stream() makes an object, 3 of the 8 us of a call
        _current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda device: torch.cuda.current_stream(device).cuda_stream)
        _current_device = torch.cuda.current_device
        # of the tensors of a tuple or list; without the public function's own look at its argument, half of its 0.2 us
        _changed = getattr(torch._C, "_increment_version", torch.autograd.graph.increment_version)
        _torch = torch
    return _torch


_MESSAGES = {-1: "bad argument", -2: f"a size beyond the limits (vocabulary {MAX_VOCAB}, top {MAX_TOP}, 2^31 rows)", -4: "out of memory",
             -5: "a CUDA call failed"}


def _refuse(message):
    raise SlaqError(-1, message)


def _check(rc, message=None):
    if rc < 0:
        raise SlaqError(rc, message or _MESSAGES.get(rc, "error"))
    return rc


def _vector(t, name, dtype, n, device):
    """The address of a contiguous tensor of n entries on GPU `device`; None passes."""
    at = _address(t, dtype, n, device)
    if at is False:
        _refuse(f"{name} is not a contiguous {dtype} tensor of {n} entries on GPU {device}")
    return at


def _matrix(t, name):
    """(address, type, rows, elements of a row, row stride, GPU) of a matrix whose rows' elements are neighbours."""
    kind, shape = _types.get(t.dtype), t.shape
    if len(shape) != 2 or not t.is_cuda or kind is None:
        _refuse(f"{name} is not a matrix of fp32, bf16 or fp16 on a GPU")
    rows, vocab = shape
    pitch, step = t.stride()
    if vocab < 1:
        _refuse("an empty vocabulary")
    if step != 1 and vocab > 1:
        _refuse(f"the elements of a row of {name} are not next to one another")
    return t.data_ptr(), kind, rows, vocab, pitch, t.get_device()


def _torch_stream(stream, device):
    """A torch stream from one or from a raw cudaStream_t.  0 is the device's default stream; torch would make a new one of it."""
    cuda = _load().cuda
    if hasattr(stream, "cuda_stream"):
        if stream.device.index != device:
            _refuse("the stream is another GPU's than the tensors")
        return stream
    return cuda.ExternalStream(stream, device=device) if stream else cuda.default_stream(device)


@contextlib.contextmanager
def _elsewhere(stream, device):
    """Another stream than torch's current one, or another device, as the current ones: what is allocated there belongs there."""
    cuda = _load().cuda
    with cuda.device(device):
        if stream is None:
            yield
        else:
            with cuda.stream(_torch_stream(stream, device)):
                yield


def _is_here(stream, device):
    return stream is None and device == _current_device()


class TokenLogprobs(NamedTuple):
    logprob: object          # [rows] float32, None without targets
    entropy: object          # [rows] float32
    norm: object             # [rows, 2] float32: largest logit, sum of exp(scale (x - largest)); for token_logprobs_grad
    top_ids: object          # [rows, top] int32, None without top
    top_logprobs: object     # [rows, top] float32


def token_logprobs(logits, targets=None, top: int = 0, scale: float = 1.0, stream=None) -> TokenLogprobs:
    """slaq_token_logprobs: ``logits`` [rows, vocab] fp32 / bf16 / fp16 with any row stride, ``targets`` int64 [rows] (negative:
    the row is not asked for) or None, ``top`` alternatives (0 .. 32), ``scale`` the inverse temperature."""
    torch = _load()
    x, kind, rows, vocab, pitch, gpu = _matrix(logits, "logits")
    if not _is_here(stream, gpu):
        with _elsewhere(stream, gpu):
            return token_logprobs(logits, targets, top, scale)
    t = _vector(targets, "targets", torch.int64, rows, gpu)
    if not 0 <= top <= MAX_TOP:
        raise SlaqError(-1 if top < 0 else -2, f"top is 0 .. {MAX_TOP}")
    empty, device, f32 = torch.empty, logits.device, torch.float32
    logprob = None if t is None else empty(rows, device=device, dtype=f32)
    entropy, norm = empty(rows, device=device, dtype=f32), empty(rows, 2, device=device, dtype=f32)
    ids = best = to_ids = to_best = None
    if top:
        ids, best = empty(rows, top, device=device, dtype=torch.int32), empty(rows, top, device=device, dtype=f32)
        to_ids, to_best = ids.data_ptr(), best.data_ptr()
    rc = _calls.token_logprobs(_at["token_logprobs"], x, kind, rows, vocab, pitch, t, scale, None if t is None else logprob.data_ptr(),
                               entropy.data_ptr(), norm.data_ptr(), top, to_ids, to_best, _current_stream(gpu))
    if rc < 0:
        _check(rc)
    return TokenLogprobs(logprob, entropy, norm, ids, best)


def _gradient(out, logits):
    """(the gradient's tensor, its address, its row stride)"""
    if out is None:
        out = _load().empty(logits.shape, dtype=logits.dtype, device=logits.device)
    elif out is not logits:
        if out.shape != logits.shape or out.dtype is not logits.dtype or out.get_device() != logits.get_device() or (out.stride(1) != 1 and out.shape[1] > 1):
            _refuse("out is not a matrix like logits with its rows' elements next to one another")
    return out, out.data_ptr(), out.stride(0)


_GRADIENT = "bad argument: a missing input, a scale that is not positive, or a gradient that overlaps the logits otherwise than row for row"


def token_logprobs_grad(logits, targets, norm, grad_logprob, entropy=None, grad_entropy=None, scale: float = 1.0, out=None, stream=None):
    """slaq_token_logprobs_grad: gradient of sum(grad_logprob x logprob + grad_entropy x entropy) by the logits, from what
    ``token_logprobs`` returned.  ``out`` may be ``logits`` itself."""
    torch = _load()
    x, kind, rows, vocab, pitch, gpu = _matrix(logits, "logits")
    if not _is_here(stream, gpu):
        with _elsewhere(stream, gpu):
            return token_logprobs_grad(logits, targets, norm, grad_logprob, entropy, grad_entropy, scale, out)
    f32 = torch.float32
    t = _vector(targets, "targets", torch.int64, rows, gpu)
    n, g = _vector(norm, "norm", f32, 2 * rows, gpu), _vector(grad_logprob, "grad_logprob", f32, rows, gpu)
    e, h = _vector(entropy, "entropy", f32, rows, gpu), _vector(grad_entropy, "grad_entropy", f32, rows, gpu)
    given = out is not None
    out, to, to_pitch = _gradient(out, logits)
    rc = _calls.token_logprobs_grad(_at["token_logprobs_grad"], x, kind, rows, vocab, pitch, t, scale, n, e, g, h, to, to_pitch, _current_stream(gpu))
    if rc < 0:
        _check(rc, _GRADIENT if rc == -1 else None)
    if given:
        _changed((out,))
    return out


def token_loss(logits, targets, row_grad, scale: float = 1.0, out=None, stream=None):
    """slaq_token_loss: (log probabilities, gradient of sum(row_grad x logprob) by the logits) in one call."""
    torch = _load()
    x, kind, rows, vocab, pitch, gpu = _matrix(logits, "logits")
    if not _is_here(stream, gpu):
        with _elsewhere(stream, gpu):
            return token_loss(logits, targets, row_grad, scale, out)
    t, g = _vector(targets, "targets", torch.int64, rows, gpu), _vector(row_grad, "row_grad", torch.float32, rows, gpu)
    given = out is not None
    out, to, to_pitch = _gradient(out, logits)
    logprob = torch.empty(rows, device=out.device, dtype=torch.float32)
    rc = _calls.token_loss(_at["token_loss"], x, kind, rows, vocab, pitch, t, scale, g, logprob.data_ptr(), to, to_pitch, _current_stream(gpu))
    if rc < 0:
        _check(rc, _GRADIENT if rc == -1 else None)
    if given:
        _changed((out,))
    return logprob, out


def _job_offsets(offsets, gpu):
    """(jobs, address): at least one entry on the GPU that the rows are on."""
    if gpu < 0:
        _refuse("the rows are not on a GPU")
    n = offsets.numel() - 1
    if n < 0:
        _refuse("offsets has no entry")
    return n, _vector(offsets, "offsets", _load().int64, n + 1, gpu)


def job_row_grad(offsets, targets=None, weights=None, out=None, stream=None):
    """slaq_job_row_grad: the derivative of each job's mean loss by the log probability of each of its rows (float32 [rows]).
    ``offsets`` int64 [jobs + 1]; rows that are no job's (before the first, behind the last, or a job's whose offsets fall or leave the
    rows) keep what ``out`` holds (without ``out``: 0)."""
    torch = _load()
    known = targets if targets is not None else weights if weights is not None else out
    if known is None:
        _refuse("the number of rows follows from targets, weights or out: one of them is wanted")
    rows, gpu = known.numel(), known.get_device()
    n, off = _job_offsets(offsets, gpu)
    if not _is_here(stream, gpu):
        with _elsewhere(stream, gpu):
            return job_row_grad(offsets, targets, weights, out)
    t, w, fresh = _vector(targets, "targets", torch.int64, rows, gpu), _vector(weights, "weights", torch.float32, rows, gpu), out is None
    if fresh:
        out = (torch.empty if n else torch.zeros)(rows, device=known.device, dtype=torch.float32)
    to = _vector(out, "out", torch.float32, rows, gpu)
    rc = _calls.job_row_grad(_at["job_row_grad"], n, off, rows, t, w, to, fresh and n > 0, _current_stream(gpu))
    if rc < 0:
        _check(rc)
    if not fresh:
        _changed((out,))
    return out


def job_losses(offsets, targets, logprob, weights=None, out=None, stream=None):
    """slaq_job_losses: float64 [jobs], the weighted mean of -logprob over each job's rows that count."""
    torch = _load()
    rows, gpu = logprob.numel(), logprob.get_device()
    n, off = _job_offsets(offsets, gpu)
    if not _is_here(stream, gpu):
        with _elsewhere(stream, gpu):
            return job_losses(offsets, targets, logprob, weights, out)
    t, lp = _vector(targets, "targets", torch.int64, rows, gpu), _vector(logprob, "logprob", torch.float32, rows, gpu)
    w = _vector(weights, "weights", torch.float32, rows, gpu)
    given = out is not None
    if not given:
        out = torch.empty(n, device=logprob.device, dtype=torch.float64)
    to = _vector(out, "out", torch.float64, n, gpu)
    rc = _calls.job_losses(_at["job_losses"], n, off, rows, t, lp, w, to, _current_stream(gpu))
    if rc < 0:
        _check(rc)
    if given:
        _changed((out,))
    return out


def append_token_losses(sched, d_job_ids, offsets, targets, logprob, weights, d_iter_times, d_cores_used, out):
    torch = _load()
    rows, gpu, n = logprob.numel(), logprob.get_device(), d_job_ids.numel()
    jobs, off = _job_offsets(offsets, gpu)
    if jobs != n:
        _refuse("offsets has one entry more than there are jobs")
    if gpu != _current_device():
        _refuse("the rows are on another GPU than the current one, which is the handle's")
    t, lp = _vector(targets, "targets", torch.int64, rows, gpu), _vector(logprob, "logprob", torch.float32, rows, gpu)
    w = _vector(weights, "weights", torch.float32, rows, gpu)
    given = out is not None
    if not given:        # its memory is the handle's stream's: not in use by earlier work of torch's, nor given to later work too early
        with contextlib.nullcontext() if sched._stream == _current_stream(gpu) else _elsewhere(sched._stream, gpu):
            out = torch.empty(n, dtype=torch.float64, device=logprob.device)
    sched._check(sched._lib.slaq_append_token_losses(
        sched._h, n, _vector(d_job_ids, "job ids", torch.int32, n, gpu), off, rows, t, lp, w,
        _vector(d_iter_times, "iteration times", torch.float64, n, gpu), _vector(d_cores_used, "cores", torch.int32, n, gpu),
        _vector(out, "out", torch.float64, n, gpu)))
    if given:
        _changed((out,))
    return out


class _Tensor(ctypes.Structure):
    _fields_ = [("param", c_void_p), ("grad", c_void_p), ("master", c_void_p), ("exp_avg", c_void_p), ("exp_avg_sq", c_void_p),
                ("exp_avg_scale", c_void_p), ("exp_avg_sq_scale", c_void_p), ("n", c_int64), ("group", c_int32), ("reserved", c_int32)]


class _Group(ctypes.Structure):
    _fields_ = [("lr", c_double), ("beta1", c_double), ("beta2", c_double), ("eps", c_double), ("weight_decay", c_double),
                ("grad_scale", c_double), ("step", c_int64)]


def _group(lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, grad_scale=1.0, step=0):
    if not -1 <= step <= 1 << 53:      # the field would hold another number
        _refuse("a count of steps is 0 .. 2^53")
    return _Group(lr, betas[0], betas[1], eps, weight_decay, grad_scale, step)


class AdamW:
    """A plan of slaq_adamw_*: one step over all tensors is one launch.

    ``params`` and ``grads``: lists of contiguous CUDA tensors (fp32, bf16 or fp16; gradients of the weights' type or fp32);
    ``group_of``: the group of each tensor (default: all 0); ``groups``: a list of dicts with ``lr``, ``betas``, ``eps``,
    ``weight_decay``, ``grad_scale``, ``step`` (any may be left out; ``eps`` is 0 or at least 2^-126, and with 0 an element whose
    second moment is 0 becomes NaN, as the formula says).  ``masters``: fp32 copies that the step works on, the
    weights being their rounding.  ``state_bits`` 32 (fp32 states) or 8 (float8_e4m3fn codes with a float32 scale per 256
    elements, the second moment as its square root).  States are made as zeros, or taken over as lists: ``exp_avg``,
    ``exp_avg_sq`` and, in 8 bits, ``exp_avg_scale``, ``exp_avg_sq_scale``; they are attributes of the same names."""

    def __init__(self, params, grads, group_of=None, groups=None, state_bits: int = 32, masters=None, exp_avg=None, exp_avg_sq=None,
                 exp_avg_scale=None, exp_avg_sq_scale=None, stream=None):
        torch = _load()
        self._h = c_void_p()
        self._lib = load_library()
        params, n = list(params), len(params)
        if not params:
            _refuse("a plan without tensors")
        device, kind = params[0].device, params[0].dtype
        if state_bits not in (8, 32):
            _refuse("states are kept in 8 or in 32 bits")
        state, eight = (torch.float8_e4m3fn, True) if state_bits == 8 else (torch.float32, False)
        group_of = [0] * n if group_of is None else [int(g) for g in group_of]
        self._groups = [dict(g) for g in ([{}] if groups is None else groups)]
        groups = [_group(**g) for g in self._groups]
        grads = list(grads)
        if not all(0 <= g < len(groups) for g in group_of) or any(g.step < 0 for g in groups):
            _refuse("a tensor's group is not one of the groups, or a group has a negative count of steps")
        if kind not in _types or not params[0].is_cuda or len(grads) != n or len(group_of) != n or not groups:
            _refuse("parameters are fp32, bf16 or fp16 tensors on a GPU, with a gradient and a group each")

        gpu = device.index
        with contextlib.nullcontext() if _is_here(stream, gpu) else _elsewhere(stream, gpu):
            raw = _current_stream(gpu)
            def states(given, dtype, count):
                return [torch.zeros(count(p), device=device).to(dtype) for p in params] if given is None else list(given)
            blocks = lambda p: -(-p.numel() // STATE_BLOCK)   # noqa: E731
            self.exp_avg = states(exp_avg, state, lambda p: p.numel())
            self.exp_avg_sq = states(exp_avg_sq, state, lambda p: p.numel())
            self.exp_avg_scale = states(exp_avg_scale, torch.float32, blocks) if eight else None
            self.exp_avg_sq_scale = states(exp_avg_sq_scale, torch.float32, blocks) if eight else None
            self.params, self.grads, self.masters = params, grads, None if masters is None else list(masters)
            grad_kind = grads[0].dtype
            if grad_kind not in (kind, torch.float32):
                _refuse("gradients are of the parameters' type or fp32")
            lists = [("params", params, kind), ("grads", grads, grad_kind), ("masters", self.masters, torch.float32),
                     ("exp_avg", self.exp_avg, state), ("exp_avg_sq", self.exp_avg_sq, state)]
            table, sizes = (_Tensor * n)(), [p.numel() for p in params]
            for name, field, tensors, dtype in [(f, {"params": "param", "grads": "grad", "masters": "master"}.get(f, f), ts, d) for f, ts, d in lists]:
                if tensors is None:
                    continue
                if len(tensors) != n:
                    _refuse(f"{name} has another length than params")
                for row, size, t in zip(table, sizes, tensors):
                    setattr(row, field, _vector(t, name, dtype, size, gpu))
            if eight:
                for name, tensors in (("exp_avg_scale", self.exp_avg_scale), ("exp_avg_sq_scale", self.exp_avg_sq_scale)):
                    if len(tensors) != n:
                        _refuse(f"{name} has another length than params")
                    for row, size, t in zip(table, sizes, tensors):
                        setattr(row, name, _vector(t, name, torch.float32, -(-size // STATE_BLOCK), gpu))
            for row, size, k in zip(table, sizes, group_of):
                row.n, row.group = size, k
            numels = np.array(sizes, np.int64)
            need = self._lib.slaq_adamw_workspace_bytes(n, numels.ctypes.data, len(groups))
            self._ws = torch.empty(max(need, 1), dtype=torch.uint8, device=device)
            # what is the plan's own memory: torch gives it away when the streams that use it have passed
            self._own = [self._ws] + [t for given, made in ((exp_avg, self.exp_avg), (exp_avg_sq, self.exp_avg_sq), (exp_avg_scale, self.exp_avg_scale),
                                                             (exp_avg_sq_scale, self.exp_avg_sq_scale)) if given is None and made is not None for t in made]
            rc = self._lib.slaq_adamw_create(self._ws.data_ptr(), need, n, table, len(groups), (_Group * len(groups))(*groups),
                                             _types[kind], _types[grad_kind], state_bits, raw, ctypes.byref(self._h))
        _check(rc, {-1: "a group or its numbers out of range, a tensor listed twice, tensors that overlap, or a stream that is being captured"}.get(rc))
        self._gpu, self._n_groups = gpu, len(groups)
        self._streams = {raw}                       # those that it is kept for
        self._watched = [p for p in params if p.requires_grad]

    def _ok(self, rc):
        return _check(rc, self._lib.slaq_adamw_last_error(self._h).decode() if rc < 0 else None)

    def _here(self):
        """The raw current stream, for which the plan's memory is kept from now on."""
        raw = _current_stream(self._gpu)
        if raw not in self._streams:
            stream = _torch_stream(raw, self._gpu)
            for t in self._own:
                t.record_stream(stream)
            self._streams.add(raw)
        return raw

    def _run(self, stream, call):
        with contextlib.nullcontext() if _is_here(stream, self._gpu) else _elsewhere(stream, self._gpu):
            self._ok(call(self._here()))

    def step(self, active=None, stream=None):
        """One step of the groups whose entry of ``active`` (int32 CUDA tensor [groups], for instance the allocation of
        ``schedule_device``) is above 0; None: of all."""
        if not _is_here(stream, self._gpu):
            with _elsewhere(stream, self._gpu):
                return self.step(active)
        a = _vector(active, "active", _torch.int32, self._n_groups, self._gpu)
        rc = _calls.adamw_step(_at["adamw_step"], self._h.value, a, self._here())
        if rc < 0:
            self._ok(rc)
        if self._watched:
            _changed(self._watched)

    def set_group(self, group: int, stream=None, **values):
        """New numbers of a group from the next step on; what is not named stays as it is, the count of steps too."""
        if not 0 <= group < self._n_groups:
            raise SlaqError(-2, "no such group")
        merged = {**self._groups[group], **values}
        numbers = _group(**{"step": -1, **{k: v for k, v in merged.items() if k != "step"}, **values})
        self._run(stream, lambda raw: self._lib.slaq_adamw_set_group(self._h, group, ctypes.byref(numbers), raw))
        self._groups[group] = merged

    def set_grads(self, grads, stream=None):
        """Other gradient tensors of the same types and sizes from the next step on."""
        grads = list(grads)
        if len(grads) != len(self.params):
            _refuse("grads has another length than params")
        rows = (c_void_p * len(grads))(*[_vector(g, "grads", old.dtype, old.numel(), self._gpu) for g, old in zip(grads, self.grads)])
        self._run(stream, lambda raw: self._lib.slaq_adamw_set_grads(self._h, rows, raw))
        self.grads = grads

    def get_steps(self, stream=None) -> np.ndarray:
        """Steps taken per group; waits for the stream."""
        out = np.empty(self._n_groups, np.int64)
        self._run(stream, lambda raw: self._lib.slaq_adamw_get_steps(self._h, out.ctypes.data, raw))
        return out

    def close(self):
        if getattr(self, "_h", None):
            self._lib.slaq_adamw_destroy(self._h)
            self._h = c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


__all__ = ["AdamW", "TokenLogprobs", "token_logprobs", "token_logprobs_grad", "token_loss", "job_row_grad", "job_losses"]
