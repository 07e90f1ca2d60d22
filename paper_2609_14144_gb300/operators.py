"""Operators that train and score a readout, on torch CUDA tensors.

A readout is fitted by distilling the full model's answers into it and judged by
the probabilities it gives.  These calls are that program's building blocks (see
include/ee.h for the exact definitions): affine maps and RMSNorm with their
gradients, log probabilities of given tokens with the best alternatives, and
the distillation loss over a teacher's best tokens with its gradient.

Matrices are two-dimensional with unit stride along a row and any row stride.
Every call enqueues on `stream` (default: the current one), allocates what it
returns there, and does not synchronise.  Outputs passed in are written and
returned.
"""
from __future__ import annotations

import contextlib
import ctypes

import torch

from . import _lib
from ._lib import check

__all__ = ["linear", "linear_backward", "rms_norm", "rms_norm_backward", "token_logprobs", "distill_topk",
           "distill_topk_step", "distill_topk_backward"]

_TYPES = {torch.bfloat16: _lib.BF16, torch.float16: _lib.FP16, torch.float32: _lib.FP32}
_ACTS = {None: 0, "none": 0, "relu": 1, "silu": 2, "gelu": 3}


def _type(t, name: str) -> int:
    try:
        return _TYPES[t.dtype]
    except KeyError:
        raise ValueError(f"{name} must be bfloat16, float16 or float32, not {t.dtype}") from None


def _mat(t, name: str, rows=None, cols=None, dtype=None) -> int:
    """Checks a matrix and returns its row stride."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dim() != 2 or (rows is not None and t.shape[0] != rows) or (cols is not None and t.shape[1] != cols):
        raise ValueError(f"{name} must have shape [{'rows' if rows is None else rows}, "
                         f"{'width' if cols is None else cols}], not {list(t.shape)}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name} must have unit stride along its rows")
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], t.stride(0))


def _vec(t, name: str, n: int, dtype=None):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dim() != 1 or t.shape[0] != n or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{name} must be contiguous with {n} elements")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")


def _full(t, name: str, shape, dtype):
    """Checks a contiguous tensor that the caller passes for a result."""
    if not t.is_cuda or tuple(t.shape) != tuple(shape) or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} CUDA tensor of shape {list(shape)}")


@contextlib.contextmanager
def _other_device_or_stream(device, stream):
    with torch.cuda.device(device):
        if stream is None:
            yield torch.cuda.current_stream(device)
        else:
            with torch.cuda.stream(stream):
                yield stream


class _Here:
    """The common case of _on: the current device and stream."""

    def __init__(self, device):
        self.stream = torch.cuda.current_stream(device)

    def __enter__(self):
        return self.stream

    def __exit__(self, *exc):
        return False


def _on(ref, stream):
    """Context in which tensors are allocated and kernels launched: ref's
    device and the given stream, so that the memory belongs to the stream that
    uses it."""
    if stream is None and ref.device.index == torch.cuda.current_device():
        return _Here(ref.device)
    return _other_device_or_stream(ref.device, stream)


def _same_device(ref, **tensors):
    for name, t in tensors.items():
        if t is not None and t.device != ref.device:
            raise ValueError(f"{name} is on {t.device}, not {ref.device}")


def _ptr(t):
    return None if t is None else t.data_ptr()


def _scratch(nbytes: int, given, device):
    """Memory for a call's intermediate values: the caller's, if it is enough."""
    if nbytes == 0:
        return None
    if given is not None:
        if given.device != device or not given.is_contiguous() or given.numel() * given.element_size() < nbytes:
            raise ValueError(f"scratch must be a contiguous tensor of at least {nbytes} bytes on {device}")
        return given
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _activation(name) -> int:
    try:
        return _ACTS[name]
    except (KeyError, TypeError):
        raise ValueError(f"unknown activation {name!r}") from None


# ---------------------------------------------------------------- affine maps
def linear(x, w, bias=None, residual=None, activation=None, out_dtype=None, keep_preact: bool = False, out=None,
           scratch=None, stream=None):
    """act(x w^T + bias) + residual for x [rows, n_in] and w [n_out, n_in], both
    bf16 or both fp16; bias [n_out] of that type.  The result has x's type, or
    out_dtype=torch.float32; a residual has the result's.  activation: None,
    "relu", "silu" or "gelu".  keep_preact=True also returns x w^T + bias in fp32,
    which linear_backward needs behind an activation."""
    lib = _lib.load()
    ld_x = _mat(x, "x")
    rows, n_in = x.shape
    ld_w = _mat(w, "w", None, n_in, x.dtype)
    n_out = w.shape[0]
    out_dtype = out_dtype or (x.dtype if out is None else out.dtype)
    if bias is not None:
        _vec(bias, "bias", n_out, x.dtype)
    ld_r = n_out if residual is None else _mat(residual, "residual", rows, n_out, out_dtype)
    act = _activation(activation)
    _same_device(x, w=w, bias=bias, residual=residual, out=out)
    with _on(x, stream) as s:
        if out is None:
            out = torch.empty((rows, n_out), dtype=out_dtype, device=x.device)
        ld_o = _mat(out, "out", rows, n_out, out_dtype)
        pre = torch.empty((rows, n_out), dtype=torch.float32, device=x.device) if keep_preact else None
        a = _lib.LinearArgs(_type(x, "x"), _type(out, "out"), act, n_in, n_out, rows, x.data_ptr(), ld_x, w.data_ptr(),
                            ld_w, _ptr(bias), _ptr(residual), ld_r, out.data_ptr(), ld_o, _ptr(pre))
        nb = ctypes.c_size_t(0)
        check(lib.ee_linear_scratch_bytes(ctypes.byref(a), ctypes.byref(nb)))
        mem = _scratch(nb.value, scratch, x.device)
        check(lib.ee_linear(ctypes.byref(a), _ptr(mem), nb.value, s.cuda_stream))
    return (out, pre) if keep_preact else out


def linear_backward(dy, x, w, activation=None, preact=None, dx=True, dw=True, dbias=True, dw_dtype=None, scratch=None,
                    stream=None):
    """(dx, dw, dbias) of linear for dy [rows, n_out] of x's type; the residual's
    gradient is dy.  Each of dx, dw, dbias is True, False (not computed, None is
    returned) or a tensor to write.  x may be None without dw, w without dx (its
    other shape is then taken from the one given).  dw has the operands' type or
    dw_dtype=torch.float32; dbias is fp32.  Behind an activation preact is what
    linear(..., keep_preact=True) returned, and dy act'(preact) is rounded to the
    operands' type for the two products."""
    lib = _lib.load()
    ld_dy = _mat(dy, "dy")
    rows, n_out = dy.shape
    if w is None and x is None:
        raise ValueError("x or w is needed for the shape")
    n_in = (x if w is None else w).shape[-1]
    ld_x = n_in if x is None else _mat(x, "x", rows, n_in, dy.dtype)
    ld_w = n_in if w is None else _mat(w, "w", n_out, n_in, dy.dtype)
    want_dx, want_dw, want_db = (t is not None and t is not False for t in (dx, dw, dbias))
    if (want_dx and w is None) or (want_dw and x is None):
        raise ValueError("dx needs w, dw needs x")
    act = _activation(activation)
    if act:
        if preact is None:
            raise ValueError("preact is needed behind an activation")
        _full(preact, "preact", (rows, n_out), torch.float32)
    _same_device(dy, x=x, w=w, preact=preact if act else None)
    with _on(dy, stream) as s:
        if dx is True:
            dx = torch.empty((rows, n_in), dtype=dy.dtype, device=dy.device)
        if dw is True:
            dw = torch.empty((n_out, n_in), dtype=dw_dtype or dy.dtype, device=dy.device)
        if dbias is True:
            dbias = torch.empty(n_out, dtype=torch.float32, device=dy.device)
        ld_dx = _mat(dx, "dx", rows, n_in, dy.dtype) if want_dx else n_in
        if want_dw:
            _full(dw, "dw", (n_out, n_in), dw_dtype or dw.dtype)
        if want_db:
            _full(dbias, "dbias", (n_out,), torch.float32)
        dx, dw, dbias = (t if want else None for t, want in ((dx, want_dx), (dw, want_dw), (dbias, want_db)))
        _same_device(dy, dx=dx, dw=dw, dbias=dbias)
        a = _lib.LinearGradArgs(_type(dy, "dy"), act, n_in, n_out, rows, dy.data_ptr(), ld_dy, _ptr(x), ld_x, _ptr(w),
                                ld_w, _ptr(preact) if act else None, _ptr(dx), ld_dx, _ptr(dw),
                                _type(dw, "dw") if want_dw else 0, 0, _ptr(dbias))
        nb = ctypes.c_size_t(0)
        check(lib.ee_linear_backward_scratch_bytes(ctypes.byref(a), ctypes.byref(nb)))
        mem = _scratch(nb.value, scratch, dy.device)
        check(lib.ee_linear_backward(ctypes.byref(a), _ptr(mem), nb.value, s.cuda_stream))
    return dx, dw, dbias


# ---------------------------------------------------------------- RMSNorm
def rms_norm(x, gain, eps: float, out_dtype=None, out=None, stream=None):
    """(y, rstd): y = x rstd gain with rstd = 1 / sqrt(mean x^2 + eps) per row
    (fp32, for rms_norm_backward).  y has x's type, or out_dtype."""
    lib = _lib.load()
    ld_x = _mat(x, "x")
    rows, d = x.shape
    _vec(gain, "gain", d)
    out_dtype = out_dtype or (x.dtype if out is None else out.dtype)
    _same_device(x, gain=gain, out=out)
    with _on(x, stream) as s:
        if out is None:
            out = torch.empty((rows, d), dtype=out_dtype, device=x.device)
        ld_y = _mat(out, "out", rows, d, out_dtype)
        rstd = torch.empty(rows, dtype=torch.float32, device=x.device)
        check(lib.ee_rms_norm(x.data_ptr(), _type(x, "x"), rows, d, ld_x, gain.data_ptr(), _type(gain, "gain"),
                              float(eps), out.data_ptr(), _type(out, "out"), ld_y, rstd.data_ptr(), s.cuda_stream))
    return out, rstd


def rms_norm_backward(dy, x, gain, rstd, dx=True, dgain=True, scratch=None, stream=None):
    """(dx, dgain) of rms_norm: dx of x's type, dgain fp32 [d].  Each of them is
    True, False (None is returned) or a tensor to write; dx may be dy."""
    lib = _lib.load()
    ld_x = _mat(x, "x")
    rows, d = x.shape
    ld_dy = _mat(dy, "dy", rows, d)
    _vec(gain, "gain", d)
    _vec(rstd, "rstd", rows, torch.float32)
    _same_device(x, dy=dy, gain=gain, rstd=rstd)
    with _on(x, stream) as s:
        if dx is True:
            dx = torch.empty((rows, d), dtype=x.dtype, device=x.device)
        if dgain is True:
            dgain = torch.empty(d, dtype=torch.float32, device=x.device)
        dx, dgain = (None if t is False else t for t in (dx, dgain))
        ld_dx = d if dx is None else _mat(dx, "dx", rows, d, x.dtype)
        mem, nb = None, ctypes.c_size_t(0)
        if dgain is not None:
            _full(dgain, "dgain", (d,), torch.float32)
            check(lib.ee_rms_norm_scratch_bytes(rows, d, ctypes.byref(nb)))
            mem = _scratch(nb.value, scratch, x.device)
        _same_device(x, dx=dx, dgain=dgain)
        check(lib.ee_rms_norm_backward(dy.data_ptr(), _type(dy, "dy"), ld_dy, x.data_ptr(), _type(x, "x"), rows, d, ld_x,
                                       gain.data_ptr(), _type(gain, "gain"), rstd.data_ptr(), _ptr(dx), ld_dx,
                                       _ptr(dgain), _ptr(mem), nb.value, s.cuda_stream))
    return dx, dgain


# ---------------------------------------------------------------- logits
def token_logprobs(logits, ids=None, k: int = 0, temperature: float = 1.0, stream=None):
    """(logprob, entropy, lse, top_logprob, top_ids) per row of logits [rows,
    vocab], with p = softmax(logits / temperature): log p of ids (int32 [rows];
    below 0: no token, 0 is returned; None: None is returned), the entropy, log sum
    exp(logits / temperature), and the k best tokens with their log p, best first,
    equal logits by the lower index ([rows, k])."""
    lib = _lib.load()
    ld = _mat(logits, "logits")
    rows, vocab = logits.shape
    if ids is not None:
        _vec(ids, "ids", rows, torch.int32)
    _same_device(logits, ids=ids)
    with _on(logits, stream) as s:
        # one allocation: logprob, entropy, lse, top_logprob
        dev, k = logits.device, int(k)
        f = torch.empty(rows * (3 + max(k, 0)), dtype=torch.float32, device=dev)
        top_ids = torch.empty((rows, max(k, 0)), dtype=torch.int32, device=dev)
        ent, lse, lp, top = f[:rows], f[rows:2 * rows], f[2 * rows:3 * rows], f[3 * rows:].view(rows, max(k, 0))
        if ids is None:
            lp = None
        check(lib.ee_token_logprobs(logits.data_ptr(), _type(logits, "logits"), rows, vocab, ld, _ptr(ids), k,
                                    float(temperature), _ptr(lp), ent.data_ptr(), lse.data_ptr(), top.data_ptr(),
                                    top_ids.data_ptr(), s.cuda_stream))
    return lp, ent, lse, top, top_ids


def _lists(logits, ids, teacher):
    rows = logits.shape[0]
    ld_i = _mat(ids, "teacher_ids", rows, None, torch.int32)
    ld_t = _mat(teacher, "teacher", rows, ids.shape[1], torch.float32)
    _same_device(logits, teacher_ids=ids, teacher=teacher)
    return ld_i, ld_t, ids.shape[1]


def _distill(logits, ids, teacher, temperature, tail, weight, grad, want_stats, stream):
    lib = _lib.load()
    ld = _mat(logits, "logits")
    rows, vocab = logits.shape
    ld_i, ld_t, k = _lists(logits, ids, teacher)
    if weight is not None:
        _vec(weight, "weight", rows, torch.float32)
    _same_device(logits, weight=weight)
    with _on(logits, stream) as s:
        loss = torch.empty(rows, dtype=torch.float32, device=logits.device)
        stats = torch.empty((rows, 4), dtype=torch.float32, device=logits.device) if want_stats else None
        if grad is True:
            grad = torch.empty((rows, vocab), dtype=logits.dtype, device=logits.device)
        ld_g = vocab if grad is None else _mat(grad, "grad", rows, vocab, logits.dtype)
        _same_device(logits, grad=grad)
        check(lib.ee_distill_topk(logits.data_ptr(), _type(logits, "logits"), rows, vocab, ld, ids.data_ptr(), ld_i,
                                  teacher.data_ptr(), ld_t, k, float(temperature), int(bool(tail)), loss.data_ptr(),
                                  _ptr(stats), _ptr(weight), _ptr(grad), ld_g, s.cuda_stream))
    return loss, stats, grad


def distill_topk(logits, teacher_ids, teacher, temperature: float = 1.0, tail: bool = False, stream=None):
    """(loss, stats): the distillation loss per row of student logits [rows, vocab]
    against a teacher's best tokens (teacher_ids int32 and teacher fp32 [rows, k];
    an id below 0 marks an absent entry), and what distill_topk_backward needs.
    tail=False: the teacher's values are renormalised over the list (logits over
    temperature, or log probabilities).  tail=True: they are log probabilities at
    this temperature, and the rest of the vocabulary is one more outcome."""
    loss, stats, _ = _distill(logits, teacher_ids, teacher, temperature, tail, None, None, True, stream)
    return loss, stats


def distill_topk_step(logits, teacher_ids, teacher, weight=None, temperature: float = 1.0, tail: bool = False, grad=None,
                      stream=None):
    """(loss, grad): distill_topk together with weight[row] (default 1) times its
    gradient, in one pass over the logits.  grad may be the logits themselves."""
    loss, _, grad = _distill(logits, teacher_ids, teacher, temperature, tail, weight, True if grad is None else grad,
                             False, stream)
    return loss, grad


def distill_topk_backward(dloss, logits, teacher_ids, teacher, stats, temperature: float = 1.0, tail: bool = False,
                          grad=None, stream=None):
    """dloss[row] times the gradient of distill_topk's loss, from the same arguments
    and the stats it returned.  grad may be the logits themselves."""
    lib = _lib.load()
    ld = _mat(logits, "logits")
    rows, vocab = logits.shape
    ld_i, ld_t, k = _lists(logits, teacher_ids, teacher)
    _vec(dloss, "dloss", rows, torch.float32)
    _full(stats, "stats", (rows, 4), torch.float32)
    _same_device(logits, dloss=dloss, stats=stats, grad=grad)
    with _on(logits, stream) as s:
        if grad is None:
            grad = torch.empty((rows, vocab), dtype=logits.dtype, device=logits.device)
        ld_g = _mat(grad, "grad", rows, vocab, logits.dtype)
        check(lib.ee_distill_topk_backward(dloss.data_ptr(), logits.data_ptr(), _type(logits, "logits"), rows, vocab, ld,
                                           teacher_ids.data_ptr(), ld_i, teacher.data_ptr(), ld_t, k, float(temperature),
                                           int(bool(tail)), stats.data_ptr(), grad.data_ptr(), ld_g, s.cuda_stream))
    return grad
