"""Operators of the model's forward and backward -- binding of
``include/gockpt_model.h``.

``linear_cross_entropy``  the head's loss over the whole vocabulary, without
                          keeping the logits (differentiable)
``head_stats``, ``head_grad``  its halves, for ranks that split the vocabulary
``Act8``, ``act8_pack``   activations in 8 bits
``linear8``               a linear layer that keeps its input so (differentiable)
``linear8_grad_weight``   its weight's gradient
``gate8``                 a (gated) activation that keeps its inputs so
                          (differentiable)

Conventions are those of the operators around the step: checks raise ValueError
or GockptError, all arithmetic runs in the library's kernels, calls are queued on
the current torch stream, or on ``stream`` where no gradient is needed, and what
a call writes counts as changed in place and must not overlap what it reads.  With
``grad_weight`` (of the weight's shape: its part of ``Session.grad``, or an fp32
sum) the backward writes the weight's gradient there, or adds to it with
``accumulate``, and returns none for it; where the weight requires no gradient,
nothing is written.  Each backward without ``accumulate`` writes every element: of
several calls on one weight in a step all but the one whose backward runs first
(the last one made) accumulate, or the program clears the sum first and all of
them do.
"""
from __future__ import annotations

import ctypes
import functools
import math
import struct

import torch
from torch.autograd import forward_ad

from . import _check
from .ops import MATRIX, NO_PADDING, TOKEN_IDS, _changed, _dtype, _empty, _here, _matrix, _stream, _token_ids
from .ops import _lib as _ops_lib

GOCKPT_EACH, GOCKPT_SUM, GOCKPT_MEAN = 0, 1, 2
GOCKPT_SILU, GOCKPT_GELU, GOCKPT_GELU_TANH = 0, 1, 2
GOCKPT_ACT8_BLOCK = 32

_TYPES = (torch.bfloat16, torch.float16, torch.float32)
_REDUCTION = {"none": GOCKPT_EACH, "sum": GOCKPT_SUM, "mean": GOCKPT_MEAN}
_KIND = {"silu": GOCKPT_SILU, "gelu": GOCKPT_GELU, "gelu_tanh": GOCKPT_GELU_TANH}

# The structs of gockpt_model.h as packed bytes.
HEAD_END = struct.Struct("<qqfi")  # ignore_id, classes, scale, reserved; after hidden, table, targets
ACT8 = struct.Struct("<QQqq")      # codes, scales, rows, cols
HEAD_SIZE = 2 * MATRIX.size + TOKEN_IDS.size + HEAD_END.size

_P = ctypes.c_void_p
_B = ctypes.c_char_p
_SZ = ctypes.POINTER(ctypes.c_size_t)
_I = ctypes.c_int


@functools.lru_cache(maxsize=1)
def _lib():
    L = _ops_lib()
    for name, args in (
            ("gockpt_head_loss_bytes", [_B, _SZ]),
            ("gockpt_head_loss", [_B, _I, _P, _P, _P, _P, ctypes.c_size_t, _P]),
            ("gockpt_head_grad_bytes", [_B, _B, _B, _SZ]),
            ("gockpt_head_grad", [_B, _P, _I, _P, _B, _B, _I, _P, ctypes.c_size_t, _P]),
            ("gockpt_act8_pack", [_B, _B, _P]),
            ("gockpt_act8_unpack", [_B, _B, _P]),
            ("gockpt_linear8_bytes", [_B, _B, _SZ]),
            ("gockpt_linear8", [_B, _B, _B, _B, _P, ctypes.c_size_t, _P]),
            ("gockpt_linear8_grad_bytes", [_B, _B, _B, _B, _B, _SZ]),
            ("gockpt_linear8_grad", [_B, _B, _B, _B, _B, _I, _P, ctypes.c_size_t, _P]),
            ("gockpt_gate8", [_I, _B, _B, _B, _B, _B, _P]),
            ("gockpt_gate8_grad", [_I, _B, _B, _B, _B, _B, _P])):
        f = getattr(L, name)
        f.argtypes, f.restype = args, ctypes.c_int
    return L


def _workspace(like, name: str, args, stream):
    """(tensor or None, address, bytes) of a call's workspace."""
    n = ctypes.c_size_t()
    rc = getattr(_lib(), name)(*args, ctypes.byref(n))
    if rc < 0:
        _check(rc, name, None)
    n = n.value
    if n == 0:
        return None, None, 0
    t = _empty(like, (n,), torch.uint8, stream)
    return t, t.data_ptr(), n


def _differentiable(stream, a, b=None) -> bool:
    """Whether a call has to be recorded; refuses what it would answer without
    the derivative that is asked for."""
    if forward_ad._current_level >= 0 and any(t is not None and forward_ad.unpack_dual(t).tangent is not None
                                              for t in (a, b)):
        raise NotImplementedError("no forward-mode derivative")
    if not (a.requires_grad or (b is not None and b.requires_grad)) or not torch.is_grad_enabled():
        return False
    if stream is not None:
        raise ValueError("stream: for calls without a gradient")
    return True


def _once(backward):
    """once_differentiable, whose 5 us are spent only where a graph of the backward
    is asked for."""
    guarded = torch.autograd.function.once_differentiable(backward)

    @functools.wraps(backward)
    def wrapped(ctx, *grads):
        return (guarded if torch.is_grad_enabled() else backward)(ctx, *grads)
    return wrapped


def _own_rows(t, cols: int, stream):
    """t, or a copy, made on the call's stream, where its rows do not lie at one
    distance, or overlap (an expanded or transposed gradient)."""
    if t.is_contiguous():
        return t
    try:
        _, rows, n, stride, _, _ = MATRIX.unpack(_matrix(t, "", None, cols))
        if rows <= 1 or stride >= n:
            return t
    except ValueError:
        pass
    with torch.cuda.stream(stream):
        return t.contiguous()


def _refuse_leaf(t, what: str) -> None:
    """What a call writes, and which no gradient would come of."""
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{what}: requires a gradient, which the call would not give it")


def _check_grad_weight(weight, grad_weight, accumulate, device: int) -> None:
    if grad_weight is None:
        if accumulate:
            raise ValueError("accumulate: into a grad_weight")
        return
    if grad_weight.shape != weight.shape:
        raise ValueError(f"grad_weight of shape {tuple(grad_weight.shape)} for a weight of shape "
                         f"{tuple(weight.shape)}")
    if grad_weight.requires_grad:
        raise ValueError("grad_weight: requires a gradient, which the call would not give it")
    _matrix(grad_weight, "grad_weight", device)


# ---- the head's cross entropy ------------------------------------------------------


def _head(hidden, table, targets, scale, first_id, ignore_id, classes) -> tuple[int, bytes]:
    device = _here(table, "table")
    if table.dim() != 2:
        raise ValueError(f"table: expected a matrix, got shape {tuple(table.shape)}")
    if hidden.shape != (*targets.shape, table.shape[1]):
        raise ValueError(f"hidden of shape {tuple(hidden.shape)} for targets of shape {tuple(targets.shape)} and a "
                         f"table of shape {tuple(table.shape)}")
    ids = _token_ids(targets, first_id, device)
    x = _matrix(hidden, "hidden", device, table.shape[1])
    return device, x + _matrix(table, "table", None) + ids + HEAD_END.pack(
        NO_PADDING if ignore_id is None else ignore_id, classes, scale, 0)


def _reduction(reduction: str) -> int:
    r = _REDUCTION.get(reduction)
    if r is None:
        raise ValueError(f"reduction: expected 'none', 'sum' or 'mean', got {reduction!r}")
    return r


def _loss(hidden, table, targets, args, reduction: int, lse: bool, logit: bool, loss: bool, stream):
    """The outputs asked for, as float32 tensors (None where not)."""
    hidden = _own_rows(hidden, table.shape[-1], stream)
    device, head = _head(hidden, table, targets, *args)
    out = [_empty(table, targets.shape if each else (), torch.float32, stream) if wanted else None
           for wanted, each in ((loss, reduction == GOCKPT_EACH), (lse, True), (logit, True))]
    ws, ptr, size = _workspace(table, "gockpt_head_loss_bytes", (head,), stream)
    _check(_lib().gockpt_head_loss(head, reduction, *(None if t is None else t.data_ptr() for t in out), ptr, size,
                                   _stream(stream, device)), "gockpt_head_loss", None)
    return out


def linear_cross_entropy(hidden, table, targets, *, scale: float = 1.0, first_id: int = 0, ignore_id=None,
                         reduction: str = "mean", grad_weight=None, accumulate: bool = False, stream=None):
    """Cross entropy of the logits scale * hidden @ table.T against targets, in
    float32: the mean over the tokens that count (0 where none does), the sum, or
    with "none" one loss for each token.  The logits are never kept.

    hidden: (*targets.shape, dim) and table: (classes, dim), both bfloat16 or both
    float16; targets: int32 or int64.  Class v has the id first_id + v.  Targets
    that are ignore_id or no row's id are masked: loss 0, no gradient, and what
    hidden holds there does not matter.

    Differentiable in hidden and in table; grad_weight and accumulate as above."""
    r = _reduction(reduction)
    args = (scale, first_id, ignore_id, 0)
    if not _differentiable(stream, hidden, table):
        return _loss(hidden, table, targets, args, r, False, False, True, stream)[0]
    _check_grad_weight(table, grad_weight, accumulate, _here(table, "table"))
    return _LinearCrossEntropy.apply(hidden, table, targets, args, r, grad_weight, accumulate)


def head_stats(hidden, table, targets, *, scale: float = 1.0, first_id: int = 0, ignore_id=None,
               classes: int | None = None, stream=None):
    """(lse, logit) of each token, float32 and of targets' shape: the log of the
    sum of exp over this table's logits, and its target's logit, 0 where the
    target is no row of the table; zeros for masked tokens.  A rank that holds
    `classes` > rows classes' range from first_id on gives that: every target in
    [0, classes) then counts, and the ranks put together the log of the sum of exp
    of their lse and the sum of their logits.  Has no gradient of its own (see
    head_grad)."""
    return tuple(_loss(hidden.detach(), table.detach(), targets, (scale, first_id, ignore_id, classes or 0),
                       GOCKPT_EACH, True, True, False, stream)[1:])


def head_grad(hidden, table, targets, lse, grad, *, scale: float = 1.0, first_id: int = 0, ignore_id=None,
              classes: int | None = None, reduction: str = "none", grad_hidden=True, grad_weight=None,
              accumulate: bool = False, stream=None):
    """(grad_hidden, grad_weight) of linear_cross_entropy from lse (of all ranks'
    classes), given the loss's gradient: one float32 for each token with "none",
    else one element.  grad_hidden: True (allocated, of hidden's type), a tensor
    to write, or None; grad_weight: a tensor of the table's shape to write, or to
    add to with accumulate, or None.  With classes, grad_hidden is this rank's
    part of the ranks' sum."""
    r = _reduction(reduction)
    if accumulate and grad_weight is None:
        raise ValueError("accumulate: into a grad_weight")
    hidden, table = _own_rows(hidden.detach(), table.shape[-1], stream), table.detach()
    device, head = _head(hidden, table, targets, scale, first_id, ignore_id, classes or 0)
    n = 1 if r != GOCKPT_EACH else targets.numel()
    for t, size, what in ((lse, targets.numel(), "lse"), (grad, n, "grad")):
        _here(t, what, device)
        if t.dtype != torch.float32 or t.numel() != size or not t.is_contiguous():
            raise ValueError(f"{what}: expected {size} contiguous float32 elements, got {tuple(t.shape)} of {t.dtype}")
    if grad_hidden is True:
        grad_hidden = _empty(hidden, hidden.shape, hidden.dtype, stream)
    elif grad_hidden is False:
        grad_hidden = None
    elif grad_hidden is not None and grad_hidden.shape != hidden.shape:
        raise ValueError(f"grad_hidden of shape {tuple(grad_hidden.shape)} for hidden of shape {tuple(hidden.shape)}")
    if grad_weight is not None and grad_weight.shape != table.shape:
        raise ValueError(f"grad_weight of shape {tuple(grad_weight.shape)} for a table of shape {tuple(table.shape)}")
    for t, what in ((grad_hidden, "grad_hidden"), (grad_weight, "grad_weight")):
        if t is not None:
            _refuse_leaf(t, what)
    _head_grad(device, head, table, lse, grad, r, grad_hidden, grad_weight, accumulate, stream)
    _changed(tuple(t for t in (grad_hidden, grad_weight) if t is not None))
    return grad_hidden, grad_weight


def _head_grad(device: int, head: bytes, table, lse, grad, reduction: int, grad_hidden, grad_weight, accumulate: bool,
               stream) -> None:
    gx = None if grad_hidden is None else _matrix(grad_hidden, "grad_hidden", device, table.shape[1])
    gw = None if grad_weight is None else _matrix(grad_weight, "grad_weight", device)
    ws, ptr, size = _workspace(table, "gockpt_head_grad_bytes", (head, gx, gw), stream)
    _check(_lib().gockpt_head_grad(head, lse.data_ptr(), reduction, grad.data_ptr(), gx, gw, accumulate, ptr, size,
                                   _stream(stream, device)), "gockpt_head_grad", None)


class _LinearCrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, hidden, table, targets, args, reduction, grad_weight, accumulate):
        loss, lse, _ = _loss(hidden, table, targets, args, reduction, True, False, True, None)
        ctx.save_for_backward(hidden, table, targets, lse)
        ctx.args, ctx.reduction, ctx.into, ctx.accumulate = args, reduction, grad_weight, accumulate
        return loss

    @staticmethod
    @_once
    def backward(ctx, grad):
        hidden, table, targets, lse = ctx.saved_tensors
        hidden = _own_rows(hidden, table.shape[1], None)
        device, head = _head(hidden, table, targets, *ctx.args)
        gx, gw = _empty(hidden, hidden.shape, hidden.dtype, None) if ctx.needs_input_grad[0] else None, None
        if ctx.needs_input_grad[1]:
            gw = _empty(table, table.shape, table.dtype, None) if ctx.into is None else ctx.into
        _head_grad(device, head, table, lse, grad.contiguous(), ctx.reduction, gx, gw,
                   ctx.accumulate and gw is not None, None)
        if gw is ctx.into and gw is not None:
            _changed((gw,))
            gw = None
        return gx, gw, None, None, None, None, None


# ---- activations in 8 bits -----------------------------------------------------------


class Act8:
    """A tensor in 8 bits, in blocks of 32 of its last dimension: ``codes`` (int8,
    rows of whole blocks) times the powers of two of ``scales`` (uint8, the
    exponent + 127; 255: a block with an inf or NaN, which stands for NaN).  What
    it stands for, bfloat16, float16 and float32 hold exactly (float16 within its
    range)."""

    # no address among them: a copy's buffer lies elsewhere
    __slots__ = ("shape", "dtype", "rows", "cols", "blocks", "buffer")

    def __init__(self, shape, dtype, device="cuda", stream=None):
        if len(shape) == 0:
            raise ValueError("a tensor without dimensions has no blocks")
        if dtype not in _TYPES:
            raise ValueError(f"expected bfloat16, float16 or float32, got {dtype}")
        self.shape, self.dtype = torch.Size(shape), dtype
        self.cols = cols = self.shape[-1]
        self.rows = rows = math.prod(self.shape[:-1])
        self.blocks = blocks = -(-cols // GOCKPT_ACT8_BLOCK)
        n = rows * blocks
        if stream is None:
            self.buffer = torch.empty(n * (GOCKPT_ACT8_BLOCK + 1), dtype=torch.uint8, device=device)
        else:
            with torch.cuda.stream(stream):
                self.buffer = torch.empty(n * (GOCKPT_ACT8_BLOCK + 1), dtype=torch.uint8, device=device)

    @property
    def codes(self):
        n = self.rows * self.blocks * GOCKPT_ACT8_BLOCK
        return self.buffer[:n].view(torch.int8).view(self.rows, self.blocks * GOCKPT_ACT8_BLOCK)

    @property
    def scales(self):
        return self.buffer[self.rows * self.blocks * GOCKPT_ACT8_BLOCK:].view(self.rows, self.blocks)

    @property
    def nbytes(self) -> int:
        return self.rows * self.blocks * (GOCKPT_ACT8_BLOCK + 1)

    def _at(self, buffer) -> bytes:
        at = buffer.data_ptr()
        return ACT8.pack(at, at + self.rows * self.blocks * GOCKPT_ACT8_BLOCK, self.rows, self.cols)

    def _pack(self, device: int) -> bytes:
        _here(self.buffer, "Act8", device)
        return self._at(self.buffer)

    def _leave(self):
        """The buffer, for a graph to save: what is left describes it wherever the
        graph has it, and holds no memory when the graph has let it go."""
        buffer, self.buffer = self.buffer, None
        return buffer

    def unpack(self, *, out=None, dtype=None, stream=None):
        """What it stands for, in dtype (default: the packed tensor's), or in out."""
        device = _here(self.buffer, "Act8")
        if out is None:
            out = _empty(self.buffer, self.shape, self.dtype if dtype is None else dtype, stream)
        elif out.shape != self.shape or (dtype is not None and out.dtype != dtype):
            raise ValueError(f"out: expected shape {tuple(self.shape)}, got {tuple(out.shape)} of {out.dtype}")
        else:
            _refuse_leaf(out, "out")
        m = _matrix(out, "out", device, self.cols)
        _check(_lib().gockpt_act8_unpack(self._pack(device), m, _stream(stream, device)), "gockpt_act8_unpack", None)
        _changed((out,))
        return out


def act8_pack(x, *, out: Act8 | None = None, stream=None) -> Act8:
    """x (bfloat16, float16 or float32) in 8 bits.  out: an Act8 of its shape to
    write.  Has no gradient."""
    device = _here(x, "x")
    _dtype(x, "x")
    if x.dim() == 0:
        raise ValueError("x: a tensor without dimensions has no blocks")
    if out is None:
        out = Act8(x.shape, x.dtype, x.device, stream)
    elif out.shape != x.shape or out.dtype != x.dtype:
        raise ValueError(f"out: of shape {tuple(out.shape)} and {out.dtype} for x of {tuple(x.shape)} and {x.dtype}")
    x = _own_rows(x.detach(), out.cols, stream)
    _check(_lib().gockpt_act8_pack(_matrix(x, "x", None, out.cols), out._pack(device), _stream(stream, device)),
           "gockpt_act8_pack", None)
    _changed((out.buffer,))
    return out


# ---- linear layer ------------------------------------------------------------------


def _linear8(x, weight, keep: bool, stream):
    device = _here(weight, "weight")
    if weight.dim() != 2:
        raise ValueError(f"weight: expected a matrix, got shape {tuple(weight.shape)}")
    rows, cols = weight.shape
    if x.dim() == 0 or x.shape[-1] != cols:
        raise ValueError(f"x of shape {tuple(x.shape)} for a weight of shape {tuple(weight.shape)}")
    x = _own_rows(x, cols, stream)
    mx, mw = _matrix(x, "x", device, cols), _matrix(weight, "weight", None)
    ws, ptr, size = _workspace(weight, "gockpt_linear8_bytes", (mx, mw), stream)
    out = _empty(x, (*x.shape[:-1], rows), x.dtype, stream)
    kept = Act8(x.shape, x.dtype, x.device, stream) if keep else None
    _check(_lib().gockpt_linear8(mx, mw, _matrix(out, "out", None, rows),
                                 None if kept is None else kept._at(kept.buffer), ptr, size,
                                 _stream(stream, device)), "gockpt_linear8", None)
    return out, kept


def _linear8_grad(grad_out, weight, kept, grad_x, grad_weight, accumulate, stream):
    device = _here(grad_out, "grad_out")
    rows = grad_out.shape[-1]
    grad_out = _own_rows(grad_out, rows, stream)
    args = (_matrix(grad_out, "grad_out", None, rows), None if weight is None else _matrix(weight, "weight", device),
            kept,
            None if grad_x is None else _matrix(grad_x, "grad_x", device, grad_x.shape[-1]),
            None if grad_weight is None else _matrix(grad_weight, "grad_weight", device))
    ws, ptr, size = _workspace(grad_out, "gockpt_linear8_grad_bytes", args, stream)
    _check(_lib().gockpt_linear8_grad(*args, accumulate, ptr, size, _stream(stream, device)), "gockpt_linear8_grad",
           None)
    _changed(tuple(t for t in (grad_x, grad_weight) if t is not None))


def linear8(x, weight, *, grad_weight=None, accumulate: bool = False, stream=None):
    """x @ weight.T for x of shape (..., cols) and weight (rows, cols), both
    bfloat16 or both float16.  For its weight's gradient it keeps x in 8 bits,
    33/32 bytes an element, and takes the gradient as grad_out.T @ what that
    stands for; the output and x's gradient are those of x itself.
    grad_weight and accumulate as above."""
    if not _differentiable(stream, x, weight):
        return _linear8(x, weight, False, stream)[0]
    _check_grad_weight(weight, grad_weight, accumulate, _here(weight, "weight"))
    return _Linear8.apply(x, weight, grad_weight, accumulate)


def linear8_grad_weight(grad_out, kept: Act8, grad_weight, *, accumulate: bool = False, stream=None):
    """grad_weight = grad_out.T @ what kept stands for, summed in fp32 and rounded
    once, or with accumulate that added to what grad_weight holds.  grad_out:
    (*kept.shape[:-1], rows), bfloat16 or float16; kept is taken in that type
    (which for float16 may have less range than what was packed)."""
    if grad_out.shape[:-1] != kept.shape[:-1] or grad_out.dim() == 0:
        raise ValueError(f"grad_out of shape {tuple(grad_out.shape)} for an input of shape {tuple(kept.shape)}")
    if grad_weight.shape != (grad_out.shape[-1], kept.cols):
        raise ValueError(f"grad_weight of shape {tuple(grad_weight.shape)}, expected "
                         f"{(grad_out.shape[-1], kept.cols)}")
    _refuse_leaf(grad_weight, "grad_weight")
    _linear8_grad(grad_out.detach(), None, kept._pack(_here(grad_out, "grad_out")), None, grad_weight, accumulate,
                  stream)
    return grad_weight


class _Linear8(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, grad_weight, accumulate):
        out, kept = _linear8(x, weight, ctx.needs_input_grad[1], None)
        # the weight is read again for x's gradient alone
        ctx.save_for_backward(weight if ctx.needs_input_grad[0] else None, None if kept is None else kept._leave())
        ctx.kept, ctx.into, ctx.accumulate = kept, grad_weight, accumulate
        ctx.x = (x.shape, x.dtype)
        ctx.weight = (weight.shape, weight.dtype)
        return out

    @staticmethod
    @_once
    def backward(ctx, grad_out):
        weight, buffer = ctx.saved_tensors
        gx = gw = None
        if ctx.needs_input_grad[0]:
            gx = torch.empty(ctx.x[0], dtype=ctx.x[1], device=grad_out.device)
        if ctx.needs_input_grad[1]:
            gw = ctx.into
            if gw is None:
                gw = torch.empty(ctx.weight[0], dtype=ctx.weight[1], device=grad_out.device)
        _linear8_grad(grad_out, weight, None if buffer is None else ctx.kept._at(buffer), gx, gw,
                      ctx.accumulate and ctx.into is not None, None)
        return gx, gw if ctx.into is None else None, None, None


# ---- activation ----------------------------------------------------------------------


def _kind(kind: str) -> int:
    k = _KIND.get(kind)
    if k is None:
        raise ValueError(f"kind: expected 'silu', 'gelu' or 'gelu_tanh', got {kind!r}")
    return k


def _gate8(x, factor, kind: int, keep: bool, stream):
    device = _here(x, "x")
    if x.dim() == 0:
        raise ValueError("x: a tensor without dimensions has no blocks")
    if factor is not None and (factor.shape != x.shape or factor.dtype != x.dtype):
        raise ValueError(f"factor of shape {tuple(factor.shape)} and {factor.dtype} for x of {tuple(x.shape)} and "
                         f"{x.dtype}")
    cols = x.shape[-1]
    x = _own_rows(x, cols, stream)
    mx, mf = _matrix(x, "x", None, cols), None
    if factor is not None:
        factor = _own_rows(factor, cols, stream)
        mf = _matrix(factor, "factor", device, cols)
    out = _empty(x, x.shape, x.dtype, stream)
    kept = [Act8(x.shape, x.dtype, x.device, stream) if keep and t is not None else None for t in (x, factor)]
    _check(_lib().gockpt_gate8(kind, mx, mf, _matrix(out, "out", None, cols),
                               *(None if k is None else k._at(k.buffer) for k in kept), _stream(stream, device)),
           "gockpt_gate8", None)
    return out, kept


def gate8(x, factor=None, *, kind: str = "silu", stream=None):
    """act(x) * factor, or act(x) without a factor, for x and factor of one shape
    and type (bfloat16, float16 or float32); kind: "silu", "gelu" (with erf) or
    "gelu_tanh".  For the gradients it keeps x and factor in 8 bits and takes both
    as what that stands for; the output is that of x and factor themselves."""
    k = _kind(kind)
    if not _differentiable(stream, x, factor):
        return _gate8(x, factor, k, False, stream)[0]
    return _Gate8.apply(x, factor, k)


class _Gate8(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, factor, kind):
        out, kept = _gate8(x, factor, kind, True, None)
        ctx.save_for_backward(*(None if k is None else k._leave() for k in kept))
        ctx.kept, ctx.kind = kept, kind
        return out

    @staticmethod
    @_once
    def backward(ctx, grad_out):
        buffers = ctx.saved_tensors
        device = _here(grad_out, "grad_out")
        cols = grad_out.shape[-1]
        grad_out = _own_rows(grad_out, cols, None)
        grads = [torch.empty(grad_out.shape, dtype=grad_out.dtype, device=grad_out.device) if needed else None
                 for needed in ctx.needs_input_grad[:2]]
        _check(_lib().gockpt_gate8_grad(ctx.kind, _matrix(grad_out, "grad_out", None, cols),
                                        *(None if k is None else k._at(b) for k, b in zip(ctx.kept, buffers)),
                                        *(None if g is None else _matrix(g, "", None, cols) for g in grads),
                                        _stream(None, device)), "gockpt_gate8_grad", None)
        return grads[0], grads[1], None
