"""Operators on rows of class scores (binding of the C ABI in ``include/dtree_scores.h``).

A forest's answers in full (``Forest.classify(x, out_kind="votes_u8")``), or any classifier's
scores, cut to the best classes (``top_scores``), drawn from (``sample``), or used to teach a
student (``distill_loss`` with autograd, ``distill_grad`` in one call).

Scores are 2-D device tensors of float32, float16, bfloat16 or, as numbers of votes whose
score is their logarithm, uint8; rows may be strided, the classes of a row may not.  Every step
runs in the gfx950 kernels of ``libdscores.so``; importing this module without the built library
raises ``ImportError``.
"""
from __future__ import annotations

import ctypes
import os

import torch

from .dtree import DTreeError, _lib as _dtree_lib, _raw_device, _stream_handle

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libdscores.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        "libdscores.so is not built; run `python -m paper_1111_1373_amd.build` "
        "(the GPU library has no fallback)")

_lib = ctypes.CDLL(LIB_PATH)

MAX_CLASSES = 1 << 20
MAX_TOP = 256


class Sampling(ctypes.Structure):
    _fields_ = [("d_temperature", ctypes.c_void_p), ("d_top_k", ctypes.c_void_p),
                ("d_top_p", ctypes.c_void_p), ("d_min_p", ctypes.c_void_p),
                ("temperature", ctypes.c_float), ("top_k", ctypes.c_int32),
                ("top_p", ctypes.c_float), ("min_p", ctypes.c_float)]


_p, _i32, _i64, _f, _s = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float,
                          ctypes.c_int)
_PROTOS = {
    "ds_last_error": (ctypes.c_char_p, []),
    "ds_top_scores": (_s, [_p, _s, _i64, _i32, _i64, _i32, _p, _p, _p, _p]),
    "ds_sample": (_s, [_p, _s, _i64, _i32, _i64, _p, _p, _p, _p]),
    "ds_distill": (_s, [_p, _s, _i64, _i32, _i64, _p, _p, _i32, _f, _p, _p, _p, _p, _i64, _p,
                        _i64, _p]),
    "ds_distill_backward": (_s, [_p, _s, _i64, _i32, _i64, _p, _p, _i32, _f, _p, _p, _p, _i64,
                                 _p]),
    "ds_distill_work_bytes": (_i64, [_i64, _i32]),
}
for _name, (_res, _args) in _PROTOS.items():
    _fn = getattr(_lib, _name)
    _fn.restype = _res
    _fn.argtypes = _args


class ScoresError(DTreeError):
    """A call that libdscores refused."""

    def __init__(self, status: int, where: str):
        self.status = status
        what = _dtree_lib.dt_status_string(status).decode()
        msg = _lib.ds_last_error().decode() or what
        RuntimeError.__init__(self, "%s: %s (%s)" % (where, what, msg))


def _check(status: int, where: str):
    if status:
        raise ScoresError(status, where)


_TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2, torch.uint8: 3}


def _scores_arg(x, votes: bool):
    """(pointer, type, rows, classes, row stride) of a matrix of scores."""
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise TypeError("scores must be a CUDA (HIP) torch tensor")
    t = _TYPES.get(x.dtype)
    if t is None or (t == 3 and not votes):
        raise TypeError("scores must be float32, float16%s, not %s"
                        % (", bfloat16 or uint8" if votes else " or bfloat16", x.dtype))
    if x.dim() != 2:
        raise TypeError("scores must be 2-D")
    n, classes = x.shape
    if classes < 1:
        raise ValueError("scores need a class at least")
    ld, step = x.stride()
    if classes > 1 and step != 1:
        raise ValueError("rows of scores must be contiguous (stride(1) == 1)")
    if n > 1 and ld < classes:
        raise ValueError("rows of scores must not overlap")
    return x.data_ptr(), t, n, classes, ld if n > 1 else classes


def _vector_arg(v, what: str, shape, dtype, device):
    """A contiguous tensor that the kernels read or write."""
    if not isinstance(v, torch.Tensor) or v.dtype != dtype or v.shape != shape or \
            v.device != device or not v.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor of shape %s on %s"
                         % (what, dtype, tuple(shape), device))
    return v


class _On:
    """Runs a call on the scores' device, and allocates its results there on the call's stream.

    The results belong to the stream that the call runs on; inputs that were allocated on another
    stream are kept until this one is through with them."""

    __slots__ = ("_guard",)

    def __init__(self, x, stream, inputs):
        self._guard = None
        if stream is not None:
            if stream.device != x.device:
                raise ValueError("the stream belongs to %s, the scores to %s"
                                 % (stream.device, x.device))
            self._guard = torch.cuda.stream(stream)       # sets the stream's device too
            for t in inputs:
                if isinstance(t, torch.Tensor):
                    t.record_stream(stream)
        elif _raw_device is None or _raw_device() != x.device.index:
            self._guard = torch.cuda.device(x.device)

    def __enter__(self):
        if self._guard is not None:
            self._guard.__enter__()
        return _stream_handle(None)

    def __exit__(self, *exc):
        if self._guard is not None:
            self._guard.__exit__(*exc)
        return False


def top_scores(x, k: int, values=None, index=None, lse=None, stream=None):
    """``ds_top_scores``: the k best classes of each row, best first, as (values float32 [n, k],
    index int32 [n, k], lse float32 [n]).  Equal scores count from the lowest class; behind a row's
    last class with a score above -inf the value is -inf and the index -1.  lse is the row's
    log-sum-exp, so that exp(values - lse) are the classes' shares."""
    ptr, t, n, classes, ld = _scores_arg(x, True)
    k = int(k)
    if not 1 <= k <= min(classes, MAX_TOP):
        raise ValueError("k must be 1 .. min(classes, %d), not %d" % (MAX_TOP, k))
    for name, out, shape, dtype in (("values", values, (n, k), torch.float32),
                                    ("index", index, (n, k), torch.int32),
                                    ("lse", lse, (n,), torch.float32)):
        if out is not None:
            _vector_arg(out, name, shape, dtype, x.device)
    with _On(x, stream, (x, values, index, lse)) as s:
        if values is None:
            values = torch.empty(n, k, dtype=torch.float32, device=x.device)
        if index is None:
            index = torch.empty(n, k, dtype=torch.int32, device=x.device)
        if lse is None:
            lse = torch.empty(n, dtype=torch.float32, device=x.device)
        _check(_lib.ds_top_scores(ptr, t, n, classes, ld, k, values.data_ptr(), index.data_ptr(),
                                  lse.data_ptr(), s), "ds_top_scores")
    return values, index, lse


def sample(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, out=None, stream=None):
    """``ds_sample``: one class drawn from each row (int32 [n], -1 for a row without a score above
    -inf), the same for the same random numbers ``u`` (float32 [n], uniform in [0, 1)).

    Of each row the ``top_k`` best classes stay (0: all), of these as many of the best as make up
    the share ``top_p`` of their weight e^(score / temperature), of these those of at least
    ``min_p`` times the best one's weight.  The class is the first up to which, in the order of
    the classes, the weights that stay sum up to more than u times their sum.  Temperature 0
    takes the best class.  Each setting is a number, or a tensor [n] (float32; top_k int32) with
    a setting for each row."""
    ptr, t, n, classes, ld = _scores_arg(x, True)
    _vector_arg(u, "u", (n,), torch.float32, x.device)
    if out is not None:
        _vector_arg(out, "out", (n,), torch.int32, x.device)
    s = Sampling()
    settings = (("temperature", temperature, torch.float32), ("top_k", top_k, torch.int32),
                ("top_p", top_p, torch.float32), ("min_p", min_p, torch.float32))
    for name, v, dtype in settings:
        if isinstance(v, torch.Tensor):
            setattr(s, "d_" + name, _vector_arg(v, name, (n,), dtype, x.device).data_ptr() or None)
        elif name == "top_k":
            if not 0 <= int(v) < 1 << 31:
                raise ValueError("top_k must be >= 0 and below 2^31, not %r" % (v,))
            s.top_k = int(v)
        else:
            setattr(s, name, float(v))
    with _On(x, stream, (x, u, temperature, top_k, top_p, min_p, out)) as raw:
        if out is None:
            out = torch.empty(n, dtype=torch.int32, device=x.device)
        _check(_lib.ds_sample(ptr, t, n, classes, ld, u.data_ptr(), ctypes.byref(s),
                              out.data_ptr(), raw), "ds_sample")
    return out


def _teacher_arg(x, values, index):
    n = x.shape[0]
    if not isinstance(values, torch.Tensor) or values.dim() != 2 or values.shape[0] != n or \
            not 1 <= values.shape[1] <= MAX_TOP:
        raise ValueError("the teacher's values must be [%d, k] with 1 <= k <= %d" % (n, MAX_TOP))
    _vector_arg(values, "values", values.shape, torch.float32, x.device)
    _vector_arg(index, "index", values.shape, torch.int32, x.device)
    return values.shape[1]


def _loss(rows, x, values, index, k, temperature, g, grad, ld_grad, s):
    """ds_distill on stream s, for arguments that are checked: loss and stats."""
    ptr, t, n, classes, ld = rows
    loss = torch.empty(n, dtype=torch.float32, device=x.device)
    stats = torch.empty(n, 2, dtype=torch.float32, device=x.device)
    need = _lib.ds_distill_work_bytes(n, classes)
    # a workspace of the call's own: calls on several streams, or graphs, never share one
    work = torch.empty(need, dtype=torch.uint8, device=x.device) if need else None
    status = _lib.ds_distill(ptr, t, n, classes, ld, values.data_ptr(), index.data_ptr(), k,
                             temperature, None if g is None else g.data_ptr(), loss.data_ptr(),
                             stats.data_ptr(), None if grad is None else grad.data_ptr(), ld_grad,
                             None if work is None else work.data_ptr(), need, s)
    if status:
        _check(status, "ds_distill")
    return loss, stats


def _gradient(rows, values, index, k, temperature, stats, g, grad, ld_grad, s):
    """ds_distill_backward on stream s, for arguments that are checked."""
    ptr, t, n, classes, ld = rows
    status = _lib.ds_distill_backward(ptr, t, n, classes, ld, values.data_ptr(), index.data_ptr(), k,
                                      temperature, stats.data_ptr(), g.data_ptr(), grad.data_ptr(),
                                      ld_grad, s)
    if status:
        _check(status, "ds_distill_backward")


def _grad_out(x, out):
    if out is not None and (not isinstance(out, torch.Tensor) or out.shape != x.shape or
                            out.dtype != x.dtype or out.device != x.device):
        raise ValueError("out must be a %s tensor of shape %s on %s"
                         % (x.dtype, tuple(x.shape), x.device))
    if out is not None and out.numel() and x.untyped_storage().data_ptr() == \
            out.untyped_storage().data_ptr():
        lo, hi = sorted((x, out), key=lambda t: t.data_ptr())
        size, ld = lo.element_size(), lo.stride(0)
        off = hi.data_ptr() - lo.data_ptr()
        # columns of one matrix lie beside each other
        beside = ld == hi.stride(0) and ld > 0 and \
            lo.shape[1] <= off % (ld * size) // size <= ld - lo.shape[1]
        if off < size * ((lo.shape[0] - 1) * ld + lo.shape[1]) and not (lo.shape[0] > 1 and beside):
            raise ValueError("out must not overlap the scores, which are read again")


def distill_grad(x, values, index, grad_loss, temperature: float = 1.0, out=None, stream=None):
    """``ds_distill``: loss (float32 [n]) and gradient of the rows of a student's scores ``x`` in
    one call, for the weights ``grad_loss`` (float32 [n]) that the rows' losses have.  Arguments
    otherwise as ``distill_loss``; ``out`` takes the gradient (x's type and shape)."""
    rows = _scores_arg(x, False)
    k = _teacher_arg(x, values, index)
    _vector_arg(grad_loss, "grad_loss", (rows[2],), torch.float32, x.device)
    _grad_out(x, out)
    with _On(x, stream, (x, values, index, grad_loss, out)) as s:
        if out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        loss, _ = _loss(rows, x, values, index, k, float(temperature), grad_loss, out,
                        _scores_arg(out, False)[4], s)
    return loss, out


def distill_forward(x, values, index, temperature: float = 1.0, stream=None):
    """``ds_distill`` without a gradient: (loss, stats); ``distill_backward`` takes the stats."""
    rows = _scores_arg(x, False)
    k = _teacher_arg(x, values, index)
    with _On(x, stream, (x, values, index)) as s:
        return _loss(rows, x, values, index, k, float(temperature), None, None, 0, s)


def distill_backward(x, values, index, stats, grad_loss, temperature: float = 1.0, out=None,
                     stream=None):
    """``ds_distill_backward``: the gradient, from the stats of ``distill_forward``."""
    rows = _scores_arg(x, False)
    k = _teacher_arg(x, values, index)
    _vector_arg(stats, "stats", (rows[2], 2), torch.float32, x.device)
    _vector_arg(grad_loss, "grad_loss", (rows[2],), torch.float32, x.device)
    _grad_out(x, out)
    with _On(x, stream, (x, values, index, stats, grad_loss, out)) as s:
        if out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        _gradient(rows, values, index, k, float(temperature), stats, grad_loss, out,
                  _scores_arg(out, False)[4], s)
    return out


class _Distill(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, values, index, temperature, rows, k):
        with _On(x, None, ()) as s:
            loss, stats = _loss(rows, x, values, index, k, temperature, None, None, 0, s)
        ctx.save_for_backward(x, values, index, stats)
        ctx.temperature = temperature
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g):
        # Saved tensors need not come back where, or with the strides that, they were saved (hooks,
        # checkpointing): everything is taken from those that did.
        x, values, index, stats = ctx.saved_tensors
        # on the stream of the forward pass; g may be a broadcast number (a sum's gradient)
        with _On(x, None, ()) as s:
            n, classes = x.shape
            ld, step = x.stride()
            if step != 1 and classes > 1 or ld < classes and n > 1:
                x = x.contiguous()
                ld = classes
            values, index, stats = values.contiguous(), index.contiguous(), stats.contiguous()
            # (as _teacher_arg and _vector_arg check, whose 4 us a small call would feel)
            device, shape = x.device, values.shape
            if values.dtype != torch.float32 or index.dtype != torch.int32 or \
                    stats.dtype != torch.float32 or len(shape) != 2 or shape[0] != n or \
                    index.shape != shape or stats.shape != (n, 2) or x.dtype not in _TYPES or \
                    values.device != device or index.device != device or stats.device != device:
                raise ValueError("a saved tensor came back with another type, shape or device")
            grad = torch.empty_like(x, memory_format=torch.contiguous_format)
            _gradient((x.data_ptr(), _TYPES[x.dtype], n, classes, ld), values, index, shape[1],
                      ctx.temperature, stats, g.contiguous(), grad, classes, s)
        return grad, None, None, None, None, None


def distill_loss(x, values, index, temperature: float = 1.0):
    """Loss of each row (float32 [n]) of a student's scores ``x`` (float32, float16 or bfloat16
    [n, classes]) against a teacher's top scores: ``values`` (float32 [n, k]) of the classes
    ``index`` (int32 [n, k]), as ``top_scores`` returns them.  With p = softmax(values / t) over
    the k entries and q = softmax(x / t) over all classes, t^2 sum p (ln p - ln q).

    Entries whose index is outside the classes, or whose value is -inf, are left out; a row without
    entries has loss 0.  The temperature is positive, at most 2^60; the loss is off by about 2^-22 t^2.
    Differentiable in ``x`` (once); runs on torch's current stream."""
    rows = _scores_arg(x, False)
    k = _teacher_arg(x, values, index)
    if values.requires_grad:
        raise ValueError("a teacher takes no gradient: detach its values")
    return _Distill.apply(x, values, index, float(temperature), rows, k)
