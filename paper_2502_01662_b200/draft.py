"""ctypes binding of include/cos_draft.h: the proposer's operators.

`sample` draws draft tokens, `top_logits` lists the largest logits of a model, `distill_loss` and `distill_step` teach a
proposer from such lists.  Argument marshalling only, as in `binding`: the arithmetic happens in the CUDA library.
"""
from __future__ import annotations

import ctypes
import operator
from typing import Optional, Sequence

from .binding import COS_MAX_MODELS, COS_OK, CosVerifyError, _current_stream, _dtype_code, _memory_of, _used_here, load_call, load_library

COS_TOP_MAX = 1024
COS_DISTILL_STATISTICS = 8

EXPORTS = ("cos_sample", "cos_top_logits", "cos_distill_loss", "cos_distill_grad", "cos_distill_step")


class cos_sample_args(ctypes.Structure):
    _fields_ = [
        ("logits", ctypes.c_void_p), ("stride_row", ctypes.c_int64), ("rows", ctypes.c_int32), ("vocab", ctypes.c_int32),
        ("dtype", ctypes.c_int32), ("device", ctypes.c_int32), ("uniforms", ctypes.c_void_p),
        ("temperature", ctypes.c_float), ("top_k", ctypes.c_int32), ("top_p", ctypes.c_float), ("min_p", ctypes.c_float),
        ("row_temperature", ctypes.c_void_p), ("row_top_k", ctypes.c_void_p), ("row_top_p", ctypes.c_void_p),
        ("row_min_p", ctypes.c_void_p), ("tokens", ctypes.c_void_p), ("prob", ctypes.c_void_p), ("kept", ctypes.c_void_p),
        ("row_status", ctypes.c_void_p), ("filtered", ctypes.c_void_p), ("stride_filtered", ctypes.c_int64),
    ]


class cos_top_args(ctypes.Structure):
    _fields_ = [
        ("logits", ctypes.c_void_p), ("stride_row", ctypes.c_int64), ("rows", ctypes.c_int32), ("vocab", ctypes.c_int32),
        ("dtype", ctypes.c_int32), ("device", ctypes.c_int32), ("k", ctypes.c_int32), ("temperature", ctypes.c_double),
        ("values", ctypes.c_void_p), ("ids", ctypes.c_void_p), ("lse", ctypes.c_void_p),
    ]


class cos_distill_args(ctypes.Structure):
    _fields_ = [
        ("student", ctypes.c_void_p), ("stride_student", ctypes.c_int64), ("rows", ctypes.c_int32), ("vocab", ctypes.c_int32),
        ("dtype", ctypes.c_int32), ("device", ctypes.c_int32), ("lists", ctypes.c_int32), ("k", ctypes.c_int32),
        ("ids", ctypes.c_void_p), ("values", ctypes.c_void_p), ("lse", ctypes.c_void_p),
        ("weights", ctypes.c_float * COS_MAX_MODELS), ("temperature", ctypes.c_double), ("row_weights", ctypes.c_void_p),
        ("loss", ctypes.c_void_p), ("statistics", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("stride_grad", ctypes.c_int64),
    ]


_lib = None
_native = None      # the module of csrc/call.cpp and the addresses of the functions it calls, or False


def _library() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        lib = load_library()
        for name, args in zip(EXPORTS, (cos_sample_args, cos_top_args, cos_distill_args, cos_distill_args, cos_distill_args)):
            fn = getattr(lib, name)
            fn.argtypes = [ctypes.POINTER(args), ctypes.c_void_p]
            fn.restype = ctypes.c_int
        _lib = lib
    return _lib


def _calls():
    """The calls in native code, (module, address of each of EXPORTS): what plain tensors go through.  False where there is none."""
    global _native
    if _native is None:
        lib, call = _library(), load_call()
        _native = (call, *(ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in EXPORTS)) if call is not None else False
    return _native


def _check(lib, st: int):
    if st != COS_OK:
        raise CosVerifyError(st, lib.cos_verify_last_error(None).decode())


def _rows(t, name: str):
    """Shape and row stride of a 2-D device tensor whose rows are contiguous."""
    if t.dim() != 2:
        raise ValueError(f"{name} must be [rows, vocab], not {tuple(t.shape)}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    rows, vocab = t.shape
    if rows < 1 or vocab < 1:
        raise ValueError(f"{name} must have at least one row and one entry")
    if max(rows, vocab) > 2 ** 31 - 1:
        raise ValueError(f"{name} has more rows or entries than 32 bits count")
    if vocab > 1 and t.stride(1) != 1:
        raise ValueError(f"the vocabulary axis of {name} must be contiguous")
    return rows, vocab, t.stride(0) if rows > 1 else vocab


def _small(t, name: str, shape, dtype, device) -> int:
    """The address of a contiguous device tensor of the given shape and type."""
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {device}")
    return t.data_ptr()


def _written(torch, t):
    """A tensor of the caller's that the library writes: autograd is told, as by an operation in place."""
    torch.autograd.graph.increment_version(t)


def _stream_of(torch, device, stream, made):
    """The address of the stream of a call, whose outputs were made in its memory."""
    if stream is None:
        return _current_stream(torch, device.index)
    _used_here(torch, stream, device, made)
    return stream.cuda_stream


def sample(logits, uniforms, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, filtered=False, stream=None) -> dict:
    """cos_sample: a token for each row of `logits` [rows, vocab] from `uniforms` [rows] float32 in [0, 1).

    temperature, top_k, top_p and min_p are numbers, or device tensors [rows] (float32; top_k int32) for a batch whose rows
    have their own; temperature 0 is greedy, top_k 0, top_p 1 and min_p 0 are no limit, and they act in this order, each
    on what the one before it left.  Returns "tokens", "kept" (how many tokens the draw was among), "row_status" (all int32
    [rows]), "prob" (float32 [rows], under the law the token was drawn from) and, where `filtered` is true or a tensor that
    takes them (`logits` itself: in place), "filtered": the logits with -inf at the tokens that were not kept.  As the
    proposer's logits of a verification at the same temperature these are the law its drafts were drawn from."""
    native = _calls() if stream is None else None
    if native:
        got = native[0].sample(native[1], logits, uniforms, temperature, top_k, top_p, min_p, filtered)
        if type(got) is dict:
            return got
        if got is not None:
            _check(_lib, got)
    # (what does not fit there, and whatever there is to complain about)
    import torch
    rows, vocab, stride = _rows(logits, "logits")
    device = logits.device
    a = cos_sample_args()
    a.logits, a.stride_row, a.rows, a.vocab, a.dtype, a.device = logits.data_ptr(), stride, rows, vocab, _dtype_code(logits.dtype), device.index
    a.uniforms = _small(uniforms, "uniforms", (rows,), torch.float32, device)
    for name, v, dtype in (("temperature", temperature, torch.float32), ("top_k", top_k, torch.int32), ("top_p", top_p, torch.float32), ("min_p", min_p, torch.float32)):
        if isinstance(v, torch.Tensor):
            setattr(a, "row_" + name, _small(v, name, (rows,), dtype, device))
        else:
            setattr(a, name, v if name != "top_k" else max(-1, min(operator.index(v), 2 ** 31 - 1)))     # (a vocabulary has no more)
    with _memory_of(torch, stream):
        buf = torch.empty((4, rows), dtype=torch.int32, device=device)
        room = torch.empty((rows, vocab), dtype=logits.dtype, device=device) if filtered is True else None
    tokens, kept, status, prob = buf.unbind(0)
    out = {"tokens": tokens, "prob": prob.view(torch.float32), "kept": kept, "row_status": status}
    a.tokens, a.kept, a.row_status, a.prob = tokens.data_ptr(), kept.data_ptr(), status.data_ptr(), prob.data_ptr()
    made = [buf]
    if filtered is not False:
        if filtered is True:
            filtered = room
            made.append(room)
        r, v, a.stride_filtered = _rows(filtered, "filtered")
        if (r, v) != (rows, vocab) or filtered.dtype != logits.dtype or filtered.device != device:
            raise ValueError("filtered must be like the logits")
        a.filtered = filtered.data_ptr()
        out["filtered"] = filtered
    lib = _library()
    _check(lib, lib.cos_sample(ctypes.byref(a), _stream_of(torch, device, stream, made)))
    if filtered is not False:
        _written(torch, filtered)
    return out


def top_logits(logits, k: int, temperature: float = 1.0, stream=None) -> dict:
    """cos_top_logits: "values" (float32) and "ids" (int32), [rows, k], of the k largest logits of each row, the largest first,
    and "lse" [rows] float32, ln sum_x exp(l(x) / temperature): what `distill_loss` takes of a teacher.  A row with a NaN or +inf lists
    nothing (ids -1) and has a NaN for "lse".  The outputs carry no gradient."""
    native = _calls() if stream is None else None
    if native:
        got = native[0].top_logits(native[2], logits, k, temperature)
        if type(got) is dict:
            return got
        if got is not None:
            _check(_lib, got)
    import torch
    rows, vocab, stride = _rows(logits, "logits")
    device = logits.device
    if not 1 <= k <= min(COS_TOP_MAX, vocab):
        raise ValueError(f"k must be in [1, {min(COS_TOP_MAX, vocab)}]")
    with _memory_of(torch, stream):
        values = torch.empty((rows, k), dtype=torch.float32, device=device)
        ids = torch.empty((rows, k), dtype=torch.int32, device=device)
        lse = torch.empty((rows,), dtype=torch.float32, device=device)
    a = cos_top_args(logits.data_ptr(), stride, rows, vocab, _dtype_code(logits.dtype), device.index, k, temperature,
                     values.data_ptr(), ids.data_ptr(), lse.data_ptr())
    lib = _library()
    _check(lib, lib.cos_top_logits(ctypes.byref(a), _stream_of(torch, device, stream, (values, ids, lse))))
    return {"values": values, "ids": ids, "lse": lse}


def _distill_args(torch, student, ids, values, lse, weights, temperature) -> cos_distill_args:
    rows, vocab, stride = _rows(student, "student")
    device = student.device
    if ids.dim() not in (2, 3):
        raise ValueError("ids must be [rows, k] or [rows, lists, k]")
    lists, k = (1 if ids.dim() == 2 else ids.shape[1]), ids.shape[-1]
    if not (1 <= lists <= COS_MAX_MODELS and 1 <= lists * k <= COS_TOP_MAX):
        raise ValueError(f"up to {COS_MAX_MODELS} lists of {COS_TOP_MAX} entries together")
    a = cos_distill_args()
    a.student, a.stride_student, a.rows, a.vocab, a.dtype, a.device = student.data_ptr(), stride, rows, vocab, _dtype_code(student.dtype), device.index
    a.lists, a.k, a.temperature = lists, k, temperature
    shape = (rows, k) if ids.dim() == 2 else (rows, lists, k)
    a.ids = _small(ids, "ids", shape, torch.int32, device)
    a.values = _small(values, "values", shape, torch.float32, device)
    if lse is not None:
        a.lse = _small(lse, "lse", (rows, lists) if ids.dim() == 3 else (rows,), torch.float32, device)
    weights = (1.0,) * lists if weights is None else tuple(weights)
    if len(weights) != lists:
        raise ValueError(f"{lists} lists need {lists} weights")
    for i, w in enumerate(weights):
        a.weights[i] = w
    return a


def _loss_call(student, ids, values, lse, weights, temperature):
    import torch
    a = _distill_args(torch, student, ids, values, lse, weights, temperature)
    loss = torch.empty((a.rows,), dtype=torch.float32, device=student.device)
    statistics = torch.empty((a.rows * (COS_DISTILL_STATISTICS + a.lists * a.k),), dtype=torch.float32, device=student.device)
    a.loss, a.statistics = loss.data_ptr(), statistics.data_ptr()
    lib = _library()
    _check(lib, lib.cos_distill_loss(ctypes.byref(a), _current_stream(torch, student.device.index)))
    return loss, statistics


def _refuse_capture(torch, student):
    """A captured backward pass of a leaf whose eager graph is alive would end the process.  Whether one is can be seen in native code alone; without that none is captured."""
    if not student.requires_grad or not student.is_leaf or not torch.cuda.is_current_stream_capturing():
        return
    native = _calls()
    if not native:
        raise RuntimeError("distill_loss: a backward pass of a leaf cannot be captured without the module of csrc/call.cpp (an eager graph of it may be alive)")
    native[0].refuse_capture(student)


def _function():
    """The autograd function, made on first use (the module does not import torch)."""
    import torch
    from torch.autograd.function import once_differentiable

    class DistillLoss(torch.autograd.Function):
        @staticmethod
        def forward(ctx, student, ids, values, lse, weights, temperature):
            loss, statistics = _loss_call(student, ids, values, lse, weights, temperature)
            ctx.save_for_backward(student, ids, values, lse, statistics)
            ctx.weights, ctx.temperature = weights, temperature
            return loss

        @staticmethod
        @once_differentiable
        def backward(ctx, upstream):
            student, ids, values, lse, statistics = ctx.saved_tensors
            _refuse_capture(torch, student)
            a = _distill_args(torch, student, ids, values, lse, ctx.weights, ctx.temperature)
            upstream = upstream.contiguous()    # (an expanded scalar, of a mean or a sum)
            grad = torch.empty((a.rows, a.vocab), dtype=student.dtype, device=student.device)
            a.row_weights = upstream.data_ptr()
            a.statistics, a.grad, a.stride_grad = statistics.data_ptr(), grad.data_ptr(), a.vocab
            lib = _library()
            _check(lib, lib.cos_distill_grad(ctypes.byref(a), _current_stream(torch, student.device.index)))
            return grad, None, None, None, None, None

    return DistillLoss


_distill_function = None


def distill_loss(student, ids, values, lse=None, weights: Optional[Sequence[float]] = None, temperature: float = 1.0):
    """cos_distill_loss and, through autograd, cos_distill_grad: loss [rows] float32 of the student's logits [rows, vocab]
    against the target t = sum_g w_g p_g of its teachers' lists, sum_x t (ln t - ln q), q = softmax(student / temperature).

    `ids` int32 and `values` float32 are one teacher's list [rows, k] or [rows, lists, k], as `top_logits` makes them (an id of -1
    is an empty entry; a token that several lists name gets the sum of its shares).  With `lse` ([rows], or [rows, lists]; the
    teachers' at the same temperature) shares are probabilities and what is not listed is left out; without, each list is
    taken to be the teacher's whole distribution.  `weights` are the ensemble's.  Differentiable in the student's logits alone, once, and not in forward mode (a student with a tangent is refused).
    (Lists made under torch.inference_mode() cannot be kept for a backward pass, as of any operation; made under torch.no_grad() they can.)
    A row without entries has loss 0 and gradient 0 (so has one whose only teacher held a NaN there, and one teacher of several that did is left out: "lse" is NaN then), and a row whose upstream gradient is 0 has gradient 0, whatever its logits.
    Forward and backward may be captured into a CUDA graph; of a leaf that an eager graph on the default stream still refers to,
    the backward pass is refused there (of any leaf, where csrc/call.cpp cannot be built).  The leaves behind a student that is computed are not looked at: no eager graph of theirs
    may be alive."""
    native = _calls()
    if native:
        got = native[0].distill_loss(native[3], native[4], student, ids, values, lse, weights, temperature)
        if type(got) is int:
            _check(_lib, got)
        elif got is not None:
            return got
    import torch
    if torch.autograd.forward_ad.unpack_dual(student).tangent is not None:
        raise NotImplementedError("distill_loss has no jvp: it is not differentiable in forward mode")
    if torch.is_grad_enabled() and student.requires_grad:
        global _distill_function
        if _distill_function is None:
            _distill_function = _function()
        return _distill_function.apply(student, ids, values, lse, None if weights is None else tuple(weights), temperature)
    return _loss_call(student, ids, values, lse, weights, temperature)[0]


def distill_step(student, ids, values, row_weights, lse=None, weights: Optional[Sequence[float]] = None, temperature: float = 1.0,
                 grad=None, stream=None) -> dict:
    """cos_distill_step: "loss" [rows] as of `distill_loss`, and "grad" [rows, vocab], the gradient of sum_n row_weights[n] loss[n] in
    the student's logits, reading them once; for training loops that know the weights of the rows beforehand
    (1 / rows for a mean).  `grad`: a tensor that takes the gradient (`student` itself: in place)."""
    native = _calls() if stream is None and grad is None else None
    if native:
        got = native[0].distill_step(native[5], student, ids, values, lse, weights, temperature, row_weights)
        if type(got) is dict:
            return got
        if got is not None:
            _check(_lib, got)
    import torch
    a = _distill_args(torch, student, ids, values, lse, weights, temperature)
    device = student.device
    a.row_weights = _small(row_weights, "row_weights", (a.rows,), torch.float32, device)
    with _memory_of(torch, stream):
        loss = torch.empty((a.rows,), dtype=torch.float32, device=device)
        statistics = torch.empty((a.rows * (COS_DISTILL_STATISTICS + a.lists * a.k),), dtype=torch.float32, device=device)
        made = [loss]
        if grad is None:
            grad = torch.empty((a.rows, a.vocab), dtype=student.dtype, device=device)
            made.append(grad)
    rows, vocab, a.stride_grad = _rows(grad, "grad")
    if (rows, vocab) != (a.rows, a.vocab) or grad.dtype != student.dtype or grad.device != device:
        raise ValueError("grad must be like the student's logits")
    a.loss, a.statistics, a.grad = loss.data_ptr(), statistics.data_ptr(), grad.data_ptr()
    lib = _library()
    _check(lib, lib.cos_distill_step(ctypes.byref(a), _stream_of(torch, device, stream, made)))
    _written(torch, grad)
    return {"loss": loss, "grad": grad}
