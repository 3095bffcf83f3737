"""Argument checks of the layer operators: the C ABI takes raw device pointers and
trusts the sizes and element types it is given, so every tensor is checked before
its address is passed on.  A failed check raises DbsError and nothing is launched."""
from __future__ import annotations

from . import _lib
from ._lib import DBS_BF16, DBS_ERR_ARG, DBS_ERR_UNSUPPORTED, DBS_F16, DbsError

CK_GROUP = _lib.DBS_CK_GROUP
MAX_DIM = 1 << 30  # of each size


def _arg_error(msg):
    return DbsError(DBS_ERR_ARG, msg)


def _choice(value, table, name):
    if value not in table:
        raise _arg_error(f"{name} is {value!r}, expected one of {', '.join(table)}")
    return table[value] if isinstance(table, dict) else value


def _dtype_code(torch, t, name):
    if t is None:
        raise _arg_error(f"{name} is required")
    if t.dtype == torch.bfloat16:
        return DBS_BF16
    if t.dtype == torch.float16:
        return DBS_F16
    raise _arg_error(f"{name} has dtype {t.dtype}, expected torch.float16 or torch.bfloat16")


def _too_large(shape, name):
    """(Sizes are handed on as 32-bit numbers, which would drop the upper bits.)"""
    return DbsError(DBS_ERR_UNSUPPORTED, f"{name} has shape {tuple(shape)}: size above 2^30")


def check_rows(t, name, dtype, device, rows, cols):
    """One 2-D tensor argument of rows x cols (None: any) of `dtype` on `device`
    with unit column stride; the elements from row to row."""
    if t is None:
        raise _arg_error(f"{name} is required")
    if t.device != device:
        raise _arg_error(f"{name} is on {t.device}, expected {device}")
    if t.dtype != dtype:
        raise _arg_error(f"{name} has dtype {t.dtype}, expected {dtype}")
    if t.dim() != 2:
        raise _arg_error(f"{name} must have 2 dimensions, not {t.dim()}")
    r, c = t.shape
    if r > MAX_DIM or c > MAX_DIM:
        raise _too_large(t.shape, name)
    if (rows is not None and r != rows) or (cols is not None and c != cols):
        raise _arg_error(f"{name} has shape {tuple(t.shape)}, expected ({'any' if rows is None else rows}, "
                         f"{'any' if cols is None else cols})")
    s0, s1 = t.stride()
    if c > 1 and s1 != 1:
        raise _arg_error(f"{name} must have unit column stride, not {s1}")
    if r > 1:
        if s0 < c:
            raise _arg_error(f"{name} has {s0} elements from row to row, needs at least {c}")
        return s0
    return c


def check_vector(t, name, dtype, device, n):
    if t.device != device or t.dtype != dtype or t.dim() != 1 or t.shape[0] != n or (n > 1 and t.stride(0) != 1):
        raise _arg_error(f"{name} must be a contiguous vector of {n} {dtype} on {device}, not {tuple(t.shape)} "
                         f"{t.dtype} on {t.device} with stride {t.stride()}")


def check_checkpoint(torch, c, name, dtype, device, rows, cols):
    if rows > MAX_DIM or cols > MAX_DIM:
        raise _too_large((rows, cols), name)
    if c.dtype != dtype:
        raise _arg_error(f"{name} holds values of {c.dtype}, expected {dtype}")
    for t, part, dt, shape in ((c.codes, "codes", torch.int8, (rows, cols)),
                               (c.exponents, "exponents", torch.uint8, (rows, -(-cols // CK_GROUP)))):
        if t.device != device or t.dtype != dt or tuple(t.shape) != shape or not t.is_contiguous():
            raise _arg_error(f"the {part} of {name} must be a contiguous {dt} tensor {shape} on {device}, not "
                             f"{t.dtype} {tuple(t.shape)} on {t.device}")


def _whole(t, ld):
    """Whether the rows of a 16-bit tensor start and end at multiples of 16 bytes."""
    return t.data_ptr() % 16 == 0 and ld % 8 == 0 and t.shape[1] % 8 == 0


def _span(t):
    n = 0 if t.numel() == 0 else 1 + sum((s - 1) * st for s, st in zip(t.shape, t.stride()))
    return t.data_ptr(), t.data_ptr() + n * t.element_size()


def _side_by_side(a, b):
    """Whether two tensors are columns of one buffer that do not meet."""
    if a.dim() != 2 or b.dim() != 2 or a.stride(0) != b.stride(0) or a.element_size() != b.element_size():
        return False
    row, size = a.stride(0), a.element_size()
    far = b.data_ptr() - a.data_ptr()
    if row <= 0 or far % size:
        return False
    at = far // size % row  # where b's rows begin in a's
    return at >= a.shape[1] and at + b.shape[1] <= row


def _check_apart(out, name, inputs):
    """A caller's output buffer must not overlap an input."""
    a, b = _span(out)
    for t, what in inputs:
        if t is not None:
            c, d = _span(t)
            if a < d and c < b and not _side_by_side(out, t):
                raise _arg_error(f"{name} overlaps {what}")


_node = None


def _no_graph(torch, call, inputs, outs, by=None):
    """The outputs of a forward call of which some input requires a gradient.  Where
    autograd is on they carry a node whose backward pass raises: without one the
    gradient would be missing with no word."""
    if not torch.is_grad_enabled():
        return outs
    global _node
    if _node is None:
        class NoGraph(torch.autograd.Function):
            @staticmethod
            def forward(ctx, call, by, outs, *inputs):
                ctx.call, ctx.by = call, by
                return tuple(t.detach() for t in outs)

            @staticmethod
            def backward(ctx, *grads):
                by = ctx.by or f"its gradients are those of LayerContext.{ctx.call}_backward"
                raise DbsError(DBS_ERR_UNSUPPORTED, f"{ctx.call} builds no autograd graph; {by}")
        _node = NoGraph
    tensors = tuple(t for t in outs if isinstance(t, torch.Tensor))
    marked = iter(_node.apply(call, by, tensors, *(t for t in inputs if t is not None)))
    return tuple(next(marked) if isinstance(t, torch.Tensor) else t for t in outs)
