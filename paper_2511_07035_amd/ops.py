"""Operators around the optimizer step -- binding of ``include/gockpt_ops.h``.

``GradList``        norm and clipping of a list of gradient tensors
``embedding``       rows of a table by token id, scaled (differentiable)
``embedding_grad``  the table's gradient

Checks of shapes and types are made here or in the library and raise
ValueError or GockptError; all arithmetic runs in the library's kernels.
Calls are queued on the current torch stream, or on ``stream``; as with any
torch operation, tensors written on another stream have to be waited for.  A
Session's step runs on its ``compute`` stream: calls that read its weights or
write its gradients or its found_inf go there (``with
torch.cuda.stream(session.compute)``), or the program has each wait for the
other.  What a call writes counts as changed in place: a backward that has
saved it raises.
"""
from __future__ import annotations

import ctypes
import functools
import math
import struct

import torch
from torch.autograd import forward_ad

from . import GOCKPT_EINVAL, GockptError, _check, lib

GOCKPT_BF16, GOCKPT_FP16, GOCKPT_FP32 = 0, 1, 2
NO_PADDING = -(1 << 63)

_DTYPE = {torch.bfloat16: GOCKPT_BF16, torch.float16: GOCKPT_FP16, torch.float32: GOCKPT_FP32}
_BITS = {torch.int32: 32, torch.int64: 64}

# The structs of gockpt_ops.h as packed bytes.
GRAD_TENSOR = struct.Struct("<QQqqqii")   # data, dst, rows, cols, stride, dtype, dst_dtype
MATRIX = struct.Struct("<Qqqqii")         # data, rows, cols, stride, dtype, reserved
TOKEN_IDS = struct.Struct("<Qqqqqii")     # ids, batch, length, stride, first_id, bits, reserved
GRAD_RESULT = struct.Struct("<dfff3f")    # sumsq, norm, found_inf, coef, reserved

# torch.autograd.graph.increment_version, which takes a list alone, without its
# 0.15 us of a call's 5 to 8
_changed = torch._C._increment_version

_P = ctypes.c_void_p
_B = ctypes.c_char_p
_SZ = ctypes.POINTER(ctypes.c_size_t)
_ops = None


def _lib():
    global _ops
    if _ops is None:
        L = lib()
        for name, args in (
                ("gockpt_grads_bytes", [_B, ctypes.c_int64, _SZ]),
                ("gockpt_grads_create", [_B, ctypes.c_int64, _P, ctypes.c_size_t, _P, ctypes.POINTER(_P)]),
                ("gockpt_grads_destroy", [_P]),
                ("gockpt_grads_norm", [_P, _P, ctypes.c_double, _P, _P]),
                ("gockpt_grads_scale", [_P, _P, _P]),
                ("gockpt_grads_clip", [_P, _P, ctypes.c_double, _P, _P]),
                ("gockpt_grads_result", [_P, _P, ctypes.c_double, _P]),
                ("gockpt_scale_ptr", [_P, ctypes.POINTER(_P)]),
                ("gockpt_embedding", [_B, _B, ctypes.c_float, _B, _P]),
                ("gockpt_embedding_grad_bytes", [ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, _SZ]),
                ("gockpt_embedding_grad", [_B, _B, ctypes.c_int64, ctypes.c_float, ctypes.c_int, _B, _P,
                                           ctypes.c_size_t, _P])):
            f = getattr(L, name)
            f.argtypes, f.restype = args, ctypes.c_int
        _ops = L
    return _ops


def gockpt_scale_ptr(ctx) -> int:
    """Device address of a context's loss scale."""
    out = _P()
    _check(_lib().gockpt_scale_ptr(ctx, ctypes.byref(out)), "gockpt_scale_ptr", None)
    return out.value


@functools.lru_cache(maxsize=256)
def gockpt_embedding_grad_bytes(tokens: int, rows: int, cols: int) -> int:
    n = ctypes.c_size_t()
    _check(_lib().gockpt_embedding_grad_bytes(int(tokens), int(rows), int(cols), ctypes.byref(n)),
           "gockpt_embedding_grad_bytes", None)
    return n.value


def _here(t, what: str, device: int | None = None) -> int:
    """The current GPU (`device`, where the caller knows it), which t is on."""
    if device is None and t.is_cuda:
        device = torch.cuda.current_device()
    if not t.is_cuda or t.get_device() != device:
        raise ValueError(f"{what}: expected a tensor on the current GPU, got one on {t.device}")
    return device


def _dtype(t, what: str) -> int:
    d = _DTYPE.get(t.dtype)
    if d is None:
        raise ValueError(f"{what}: expected bfloat16, float16 or float32, got {t.dtype}")
    return d


def _stream(stream, device: int) -> int:
    # the handle alone: 0.07 us against 1.9 for a torch.cuda.Stream around it,
    # of the 5 that a whole call of the smallest size takes
    return torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream


def _capturing(stream) -> bool:
    with torch.cuda.stream(stream):
        return torch.cuda.is_current_stream_capturing()


def _rows(shape, stride):
    """(rows, cols, row stride) of elements in row-major order, or None where
    they are not rows of adjacent elements at one distance."""
    dims = []
    for n, s in zip(shape, stride):
        if n == 0:
            return 0, 0, 0
        if n == 1:
            continue
        if dims and dims[-1][1] == n * s:
            dims[-1] = (dims[-1][0] * n, s)
        else:
            dims.append((n, s))
    if not dims:
        return 1, 1, 1
    if dims[-1][1] != 1:
        dims.append((1, 1))
    if len(dims) == 1:
        return 1, dims[0][0], dims[0][0]
    if len(dims) == 2 and dims[0][1] >= dims[1][0]:
        return dims[0][0], dims[1][0], dims[0][1]
    return None


class GradResult:
    """The device-resident outcome of a norm: one-element tensors ``norm``
    (of the unscaled gradients), ``found_inf`` (1.0 or 0.0; what
    ``Session(found_inf=...)`` takes), ``coef`` (the clipping coefficient) and
    ``sumsq`` (float64, of the elements as stored: what ranks add up);
    ``largest``: the largest magnitudes of the elements that go to float16 from
    a wider type, and to bfloat16 from float32, and are too large for it
    unscaled (0: none; what ranks take the maximum of).  found_inf is 1 where an
    element is inf or NaN, and where an element times coef is rounded to inf in
    its destination."""

    def __init__(self, device="cuda"):
        self.buffer = torch.zeros(8, dtype=torch.float32, device=device)
        self.sumsq = self.buffer[:2].view(torch.float64)
        self.norm = self.buffer[2:3]
        self.found_inf = self.buffer[3:4]
        self.coef = self.buffer[4:5]
        self.largest = self.buffer[5:7]
        self.ptr, self.device = self.buffer.data_ptr(), self.buffer.get_device()

    def update(self, max_norm: float = float("inf"), scale=None, stream=None) -> "GradResult":
        """norm, found_inf and coef again from ``sumsq`` and ``largest``, after
        ranks that hold different parameters have put theirs together."""
        device = _here(self.buffer, "result")
        _changed((self.buffer,))
        s = _stream(stream, device)
        _check(_lib().gockpt_grads_result(self.ptr, _scale_ptr(scale, device, stream, s), max_norm, s),
               "gockpt_grads_result", None)
        return self


def _scale_ptr(scale, device: int, stream, raw: int):
    """Address of a one-element float32 device tensor, or of the loss scale of
    a Session, whose steps write it: the stream of the call (`raw` its handle)
    waits for those queued so far."""
    if scale is None:
        return None
    if isinstance(scale, torch.Tensor):
        if scale.dtype != torch.float32 or scale.numel() != 1:
            raise ValueError("scale: expected a one-element float32 tensor or a Session")
        _here(scale, "scale", device)
        return scale.data_ptr()
    if not hasattr(scale, "ctx"):
        raise ValueError(f"scale: expected a one-element float32 tensor or a Session, got {type(scale).__name__}")
    if scale.compute.device_index != device:
        raise ValueError(f"scale: the Session is on GPU {scale.compute.device_index}, the call on {device}")
    if scale.compute.cuda_stream != raw:
        now = torch.cuda.current_stream(device) if stream is None else stream
        if not (_capturing(now) or _capturing(scale.compute)):
            now.wait_stream(scale.compute)
    return gockpt_scale_ptr(scale.ctx)


class GradList:
    """A handle over gradient tensors (bfloat16, float16 and float32 mixed, any
    sizes, any alignment of their elements; rows may lie apart).

    out: destinations of ``clip`` and ``scale``, one for each tensor (contiguous,
    as many elements, any of the three types: views of ``Session.grad``, say);
    None, or None in a place: in place.  Writing in place also takes a tensor
    whose dimensions are permuted.  The handle keeps the tensors alive and
    holds their addresses: make a new one when they move.  Its calls use its
    workspace one at a time: a call on another stream than the last one's waits
    there for that one.  Calls recorded in a graph run whenever it is replayed:
    the program orders the replays, and keeps the list as long as the graph."""

    def __init__(self, tensors, out=None, stream=None):
        self.handle = None
        self.tensors = list(tensors)
        self.out = [None] * len(self.tensors) if out is None else list(out)
        if len(self.out) != len(self.tensors):
            raise ValueError(f"{len(self.tensors)} tensors, {len(self.out)} destinations")
        self.device = None
        table = bytearray()
        for i, (t, o) in enumerate(zip(self.tensors, self.out)):
            self.device = _here(t, f"tensor {i}", self.device)
            d = _dtype(t, f"tensor {i}")
            size = t.numel()
            r = (1, size, size) if t.is_contiguous() else _rows(t.shape, t.stride())
            if r is None and o is None:  # element by element in place: the order does not matter
                r = _rows(*zip(*sorted(zip(t.shape, t.stride()), key=lambda x: -x[1])))
            if r is None:
                raise ValueError(f"tensor {i}: shape {tuple(t.shape)} with strides {t.stride()} is not rows of "
                                 "adjacent elements")
            if o is not None:
                _here(o, f"out {i}", self.device)
                if o.numel() != size or not o.is_contiguous():
                    raise ValueError(f"out {i}: expected {t.numel()} contiguous elements, got {tuple(o.shape)}")
            table += GRAD_TENSOR.pack(t.data_ptr(), 0 if o is None else o.data_ptr(), *r, d,
                                      d if o is None else _dtype(o, f"out {i}"))
        # what clip and scale write, for _changed: a tensor for each storage's
        # version, which views share with their base
        written = [t if o is None else o for t, o in zip(self.tensors, self.out)]
        self.written = list({id(b): b for b in (w if w._base is None else w._base for w in written)}.values())
        table, n, size = bytes(table), len(self.tensors), ctypes.c_size_t()
        _check(_lib().gockpt_grads_bytes(table, n, ctypes.byref(size)), "gockpt_grads_bytes", None)
        if self.device is None:
            self.device = torch.cuda.current_device()
        with torch.cuda.stream(stream):
            self.workspace = torch.empty(size.value, dtype=torch.uint8, device=self.device)
            self.result = GradResult(self.device)
        handle = _P()
        self.last = torch.cuda.current_stream(self.device) if stream is None else stream
        self.at = self.last.cuda_stream
        self.streams = {self.at}
        _check(_lib().gockpt_grads_create(table, n, self.workspace.data_ptr(), size.value, self.at,
                                          ctypes.byref(handle)), "gockpt_grads_create", None)
        self.handle = handle.value

    def _on(self, stream) -> int:
        """The stream of a call, on the list's GPU."""
        if self.handle is None:
            raise GockptError(GOCKPT_EINVAL, "GradList", "closed")
        if torch.cuda.current_device() != self.device:
            raise ValueError(f"the list is on GPU {self.device}, which is not the current one")
        s = _stream(stream, self.device)
        if s != self.at:
            self._move(torch.cuda.current_stream(self.device) if stream is None else stream)
        return s

    def _move(self, stream) -> None:
        """To another stream than the last call's, which waits for that call."""
        if stream.cuda_stream not in self.streams:
            # the allocator gives no memory of the list away before its work there is done
            for t in (self.workspace, self.result.buffer, *self.tensors, *(o for o in self.out if o is not None)):
                t.record_stream(stream)
            self.streams.add(stream.cuda_stream)
        if _capturing(stream) or _capturing(self.last):
            return
        stream.wait_stream(self.last)
        self.last, self.at = stream, stream.cuda_stream

    def _result(self, result) -> GradResult:
        if result is None:
            return self.result
        if result.device != self.device:
            raise ValueError(f"result: on {result.buffer.device}, the list is on GPU {self.device}")
        return result

    def norm(self, max_norm: float = float("inf"), *, scale=None, result=None, stream=None) -> GradResult:
        """The norm over all tensors, divided by ``scale`` (the loss scale the
        gradients carry: a device tensor, or a Session, whose steps queued so
        far are waited for on another stream than its own), into ``result``
        (the list's own, overwritten by its next call, if None)."""
        s = self._on(stream)
        r = self._result(result)
        p = _scale_ptr(scale, self.device, stream, s)
        _check(_lib().gockpt_grads_norm(self.handle, p, max_norm, r.ptr, s), "gockpt_grads_norm", None)
        _changed((r.buffer,))
        return r

    def clip(self, max_norm: float, *, scale=None, result=None, stream=None) -> GradResult:
        """``norm``, then every element times min(1, max_norm / (norm + 1e-6))
        in place or into ``out``.  With an inf or NaN among the gradients they
        are left, or copied, as they are, and ``found_inf`` tells, as it does
        where a scaled element is beyond the range of its ``out``."""
        s = self._on(stream)
        r = self._result(result)
        p = _scale_ptr(scale, self.device, stream, s)
        _check(_lib().gockpt_grads_clip(self.handle, p, max_norm, r.ptr, s), "gockpt_grads_clip", None)
        _changed((r.buffer, *self.written))
        return r

    def scale(self, result=None, *, stream=None) -> None:
        """Every element times ``result.coef``: the second half of ``clip``."""
        s = self._on(stream)
        r = self._result(result)
        _check(_lib().gockpt_grads_scale(self.handle, r.ptr, s), "gockpt_grads_scale", None)
        _changed(self.written)

    def close(self) -> None:
        """Releases the handle.  Waits for nothing: work that calls have queued,
        on whichever stream, still runs."""
        if self.handle is not None:
            _lib().gockpt_grads_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _matrix(t, what: str, device: int | None, cols=None) -> bytes:
    """A 2-D tensor, or with cols the rows of that many elements of any; on GPU
    `device` (None: checked by the caller)."""
    if device is not None:
        _here(t, what, device)
    d = _dtype(t, what)
    shape = t.shape
    if cols is not None and len(shape) > 0 and shape[-1] == cols and t.is_contiguous():
        return MATRIX.pack(t.data_ptr(), t.numel() // cols if cols else math.prod(shape[:-1]), cols, cols, d, 0)
    if len(shape) == 2:
        (rows, n), (stride, step) = shape, t.stride()
    elif cols is not None and len(shape) > 0:
        n, step = shape[-1], t.stride(-1)
        r = _rows(shape[:-1], t.stride()[:-1])
        if n and r is not None and r[0] and r[1] != 1 and r[0] != 1:
            r = None
        if r is None:
            raise ValueError(f"{what}: shape {tuple(shape)} with strides {t.stride()} is not rows at one distance")
        rows = t.numel() // n if n else 0
        stride = r[2] if r[1] == 1 else 1
    else:
        raise ValueError(f"{what}: expected a matrix, got shape {tuple(shape)}")
    if (step != 1 and n > 1) or (cols is not None and n != cols):
        raise ValueError(f"{what}: expected rows of {cols if cols is not None else n} adjacent elements, got shape "
                         f"{tuple(shape)} with strides {t.stride()}")
    return MATRIX.pack(t.data_ptr(), rows, n, stride, d, 0)


def _token_ids(ids, first_id: int, device: int) -> bytes:
    _here(ids, "ids", device)
    bits = _BITS.get(ids.dtype)
    if bits is None:
        raise ValueError(f"ids: expected int32 or int64, got {ids.dtype}")
    if ids.is_contiguous():
        n = ids.numel()
        return TOKEN_IDS.pack(ids.data_ptr(), 1, n, n, first_id, bits, 0)
    r = _rows(ids.shape, ids.stride())
    if r is None:
        raise ValueError(f"ids: shape {tuple(ids.shape)} with strides {ids.stride()} is not rows of adjacent ids")
    return TOKEN_IDS.pack(ids.data_ptr(), *r, first_id, bits, 0)


def _empty(like, shape, dtype, stream):
    """On like's GPU, allocated for use on the stream that the call runs on."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _lookup(weight, ids, scale, out, out_dtype, first_id, stream):
    device = _here(weight, "weight")
    w, t = _matrix(weight, "weight", None), _token_ids(ids, first_id, device)
    dim = weight.shape[1]
    shape = (*ids.shape, dim)
    given = out is not None
    if not given:
        dtype = weight.dtype if out_dtype is None else out_dtype
        code = _DTYPE.get(dtype)
        if code is None:
            raise ValueError(f"out_dtype: expected bfloat16, float16 or float32, got {dtype}")
        out = _empty(weight, shape, dtype, stream)
        o = MATRIX.pack(out.data_ptr(), ids.numel(), dim, dim, code, 0)
    else:
        if out.shape != shape or (out_dtype is not None and out.dtype != out_dtype):
            raise ValueError(f"out: expected shape {shape}, got {tuple(out.shape)} of {out.dtype}")
        if out.requires_grad and torch.is_grad_enabled():
            raise ValueError("out: requires a gradient, which the call would not give it")
        o = _matrix(out, "out", device, dim)
    _check(_lib().gockpt_embedding(w, t, scale, o, _stream(stream, device)), "gockpt_embedding", None)
    if given:
        _changed((out,))
    return out


def embedding(weight, ids, *, scale: float = 1.0, out=None, out_dtype=None, first_id: int = 0, padding_id=None,
              grad_weight=None, accumulate: bool = False, stream=None):
    """scale * weight[ids - first_id] of shape (*ids.shape, dim), rounded once
    to out_dtype (default: the weight's).  Ids outside [first_id, first_id +
    rows) are masked: zeros, and no gradient.

    Differentiable in weight, with the gradient of ``embedding_grad``: returned
    to autograd in the weight's type, or, with grad_weight (of the weight's
    shape: its part of ``Session.grad``), written or accumulated there and not
    returned; where the weight requires no gradient, nothing is written.  Each
    backward writes every row of grad_weight: with several lookups of one table
    in a step, clear it first and let all of them accumulate.  Tokens with
    padding_id add no gradient.  out and stream are for calls that need no
    gradient.  The derivative along a tangent of the weight (forward mode) is the
    tangent's lookup."""
    if accumulate and grad_weight is None:
        raise ValueError("accumulate: into a grad_weight")
    # the level is -1 outside of a dual_level
    if (weight.requires_grad and torch.is_grad_enabled()) or (
            forward_ad._current_level >= 0 and forward_ad.unpack_dual(weight).tangent is not None):
        if out is not None or stream is not None:
            raise ValueError("out and stream: for calls without a gradient")
        if grad_weight is not None:
            # the backward takes the table's rows, and so which ids count, from it
            if grad_weight.shape != weight.shape:
                raise ValueError(f"grad_weight of shape {tuple(grad_weight.shape)} for a weight of shape "
                                 f"{tuple(weight.shape)}")
            _matrix(grad_weight, "grad_weight", _here(weight, "weight"))
        return _Embedding.apply(weight, ids, scale, out_dtype, first_id, padding_id, grad_weight, accumulate)
    return _lookup(weight, ids, scale, out, out_dtype, first_id, stream)


def embedding_grad(grad_out, ids, grad_weight, *, scale: float = 1.0, accumulate: bool = False, first_id: int = 0,
                   padding_id=None, workspace=None, stream=None):
    """grad_weight[v] = scale * (sum of the rows of grad_out whose id is
    first_id + v), summed in fp32 and rounded once; every row is written.  With
    accumulate the sums are added to what grad_weight holds and rows without a
    token are left alone.  workspace: a uint8 tensor of at least
    gockpt_embedding_grad_bytes(tokens, rows, dim) (None: allocated)."""
    device = _here(grad_weight, "grad_weight")
    m = _matrix(grad_weight, "grad_weight", None)
    if grad_out.shape[:-1] != ids.shape:
        raise ValueError(f"grad_out of shape {tuple(grad_out.shape)} for ids of shape {tuple(ids.shape)}")
    rows, cols = grad_weight.shape
    ptr = size = 0
    if workspace is None:
        size = gockpt_embedding_grad_bytes(ids.numel(), rows, cols)
        if size:
            workspace = _empty(grad_weight, (size,), torch.uint8, stream)
            ptr = workspace.data_ptr()
    else:
        _here(workspace, "workspace", device)
        if workspace.dtype != torch.uint8 or not workspace.is_contiguous():
            raise ValueError("workspace: expected a contiguous uint8 tensor")
        ptr, size = workspace.data_ptr(), workspace.numel()
    x, t = _matrix(grad_out, "grad_out", device, cols), _token_ids(ids, first_id, device)
    _check(_lib().gockpt_embedding_grad(x, t, NO_PADDING if padding_id is None else padding_id, scale, accumulate, m,
                                        ptr, size, _stream(stream, device)),
           "gockpt_embedding_grad", None)
    _changed((grad_weight,))
    return grad_weight


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, weight, ids, scale, out_dtype, first_id, padding_id, grad_weight, accumulate):
        ctx.save_for_backward(ids)
        ctx.save_for_forward(ids)
        ctx.out_dtype = out_dtype
        ctx.args = dict(scale=scale, first_id=first_id, padding_id=padding_id)
        ctx.into, ctx.accumulate = grad_weight, accumulate
        ctx.like = (weight.shape, weight.dtype, weight.device)
        return _lookup(weight.detach(), ids, scale, None, out_dtype, first_id, None)

    @staticmethod
    def jvp(ctx, tangent, *_):
        (ids,) = ctx.saved_tensors
        return _lookup(tangent.contiguous(), ids, ctx.args["scale"], None, ctx.out_dtype, ctx.args["first_id"], None)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_out):
        (ids,) = ctx.saved_tensors
        into = ctx.into
        if into is None:
            shape, dtype, device = ctx.like
            into = torch.empty(shape, dtype=dtype, device=device)
        embedding_grad(grad_out.contiguous(), ids, into, accumulate=ctx.accumulate and ctx.into is not None, **ctx.args)
        return (into if ctx.into is None else None,) + (None,) * 7
