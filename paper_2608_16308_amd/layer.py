"""Dense layer operators on the MI355X -- Python binding.

The linear and gated feed-forward layers that stand beside the pruned ones,
their backward passes, and 8-bit activation checkpoints (the dense-layer part
of ``include/dbspmspv.h``).  Argument marshalling only: every step runs in
the library's HIP kernels.

    ctx = LayerContext()
    h = ctx.gated(x, w_gate, w_up, act="relu")                  # serving
    y = ctx.linear(h, w_down, residual=x)
    h, gate, up = ctx.gated(x, w_gate, w_up, save="8bit")       # training
    dx, dw_gate, dw_up = ctx.gated_backward(dh, ctx.pack(x), w_gate, w_up, gate, up)
"""
from __future__ import annotations

import ctypes

from . import _lib
from ._lib import DBS_BF16, DBS_ERR_ARG, DBS_ERR_UNSUPPORTED, DBS_F16, DbsError, check

ACTS = {"none": _lib.DBS_ACT_NONE, "relu": _lib.DBS_ACT_RELU, "silu": _lib.DBS_ACT_SILU, "gelu": _lib.DBS_ACT_GELU,
        "gelu_tanh": _lib.DBS_ACT_GELU_TANH}
SAVES = ("none", "full", "8bit")
CK_GROUP = _lib.DBS_CK_GROUP
MAX_DIM = 1 << 30  # of each size
ROWS_TOKENS = 16  # forward calls of so few tokens use no workspace


class Checkpoint:
    """A 2-D activation held in 8 bits: ``codes`` int8 [rows, cols],
    ``exponents`` uint8 [rows, ceil(cols / 32)] (both contiguous device
    tensors), ``dtype`` the type of its values (float16 or bfloat16)."""

    __slots__ = ("codes", "exponents", "dtype")

    def __init__(self, codes, exponents, dtype):
        self.codes, self.exponents, self.dtype = codes, exponents, dtype

    @property
    def shape(self):
        return self.codes.shape

    @property
    def device(self):
        return self.codes.device

    def nbytes(self):
        return self.codes.numel() + self.exponents.numel()


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


def _no_graph(torch, call, inputs, outs):
    """The outputs of a forward call of which some input requires a gradient.  Where
    autograd is on they carry a node whose backward pass raises: without one the
    gradient would be missing with no word."""
    if not torch.is_grad_enabled():
        return outs
    global _node
    if _node is None:
        class NoGraph(torch.autograd.Function):
            @staticmethod
            def forward(ctx, call, outs, *inputs):
                ctx.call = call
                return tuple(t.detach() for t in outs)

            @staticmethod
            def backward(ctx, *grads):
                raise DbsError(DBS_ERR_UNSUPPORTED, f"{ctx.call} builds no autograd graph; its gradients are those of "
                                                    f"LayerContext.{ctx.call}_backward")
        _node = NoGraph
    tensors = tuple(t for t in outs if isinstance(t, torch.Tensor))
    marked = iter(_node.apply(call, tensors, *(t for t in inputs if t is not None)))
    return tuple(next(marked) if isinstance(t, torch.Tensor) else t for t in outs)


class LayerContext:
    """Workspace of one stream (default: the current one); runs the dense layer
    operators on it.

    A call is asynchronous on the context's stream.  Where that is not torch's
    current stream, outputs belong to the context's stream and inputs are
    marked as used there; the caller orders the two streams, as for any work
    on a stream of its own.  One host thread at a time may use a context.

    No call builds an autograd graph: the gradients are those of
    ``linear_backward`` and ``gated_backward``, and a result that autograd
    follows back to one of these calls raises."""

    def __init__(self, stream=None):
        import torch
        self._torch = torch
        self._h = None
        self.stream = torch.cuda.current_stream() if stream is None else stream
        self.device = self.stream.device
        self._raw = self.stream.cuda_stream
        self._fn = _lib.load()
        out = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            check(self._fn.dbs_layer_create(ctypes.c_void_p(self._raw), ctypes.byref(out)))
        self._h = out

    def __del__(self):
        h = getattr(self, "_h", None)
        if h is not None and h.value:
            self._fn.dbs_layer_destroy(h)
            self._h = None

    # -- a call: outputs are allocated and the kernels launched in here
    def _call(self, body, inputs):
        torch = self._torch
        if torch.cuda.current_stream(self.device).cuda_stream == self._raw and \
                torch.cuda.current_device() == self.device.index:
            return body()
        for t in inputs:
            if isinstance(t, Checkpoint):
                t.codes.record_stream(self.stream)
                t.exponents.record_stream(self.stream)
            elif t is not None:
                t.record_stream(self.stream)
        with torch.cuda.stream(self.stream):
            return body()

    def _held(self, v, name, dtype, rows, cols):
        """(dbs_held, whether it is a checkpoint) of a tensor or Checkpoint."""
        if isinstance(v, Checkpoint):
            check_checkpoint(self._torch, v, name, dtype, self.device, rows, cols)
            return _lib.Held(None, 0, v.codes.data_ptr(), v.exponents.data_ptr()), True
        ld = check_rows(v, name, dtype, self.device, rows, cols)
        return _lib.Held(v.data_ptr(), ld, None, None), False

    def _keep(self, save, rows, cols, dtype):
        """(what a forward pass keeps, dbs_keep or None)."""
        torch = self._torch
        if save == "none":
            return None, None
        if save == "full":
            t = torch.empty((rows, cols), dtype=dtype, device=self.device)
            return t, _lib.Held(t.data_ptr(), cols, None, None)
        c = self._new_checkpoint(rows, cols, dtype)
        return c, _lib.Held(None, 0, c.codes.data_ptr(), c.exponents.data_ptr())

    def _new_checkpoint(self, rows, cols, dtype):
        torch = self._torch
        return Checkpoint(torch.empty((rows, cols), dtype=torch.int8, device=self.device),
                          torch.empty((rows, -(-cols // CK_GROUP)), dtype=torch.uint8, device=self.device), dtype)

    # -- forward
    def _forward_work(self, gated, t, n_in, n_out, *inputs):
        """(workspace or None, its bytes, its address) for inputs (tensor, ld)
        that are not in whole 16-byte chunks."""
        if t <= ROWS_TOKENS or all(_whole(v, ld) for v, ld in inputs):
            return None, 0, None
        n = ctypes.c_size_t()
        check(self._fn.dbs_forward_work(self._h, gated, t, n_in, n_out, ctypes.byref(n)))
        if not n.value:
            return None, 0, None
        work = self._torch.empty(n.value, dtype=self._torch.uint8, device=self.device)
        return work, n.value, work.data_ptr()

    def linear(self, x, w, bias=None, act="none", residual=None, save="none", y=None):
        """y = act(x w^T + bias) + residual for x [tokens, n_in] (or one token
        [n_in]), w [n_out, n_in]; y may be preallocated, also as the residual.
        With save "full" or "8bit" returns (y, x w^T + bias as a tensor or
        Checkpoint) for ``linear_backward``."""
        act_code, save = _choice(act, ACTS, "act"), _choice(save, SAVES, "save")
        dt, dev = _dtype_code(self._torch, x, "x"), self.device
        one = x.dim() == 1
        if one:
            x = x.unsqueeze(0)
            residual = None if residual is None else residual.unsqueeze(0)
            y = None if y is None else y.unsqueeze(0)
        ldx = check_rows(x, "x", x.dtype, dev, None, None)
        t, n_in = x.shape
        ldw = check_rows(w, "w", x.dtype, dev, None, n_in)
        n_out = w.shape[0]
        if bias is not None:
            check_vector(bias, "bias", x.dtype, dev, n_out)
        ldr = 0 if residual is None else check_rows(residual, "residual", x.dtype, dev, t, n_out)
        given = y
        if y is not None:
            ldy = check_rows(y, "y", x.dtype, dev, t, n_out)
            same = residual is not None and y.data_ptr() == residual.data_ptr() and ldy == ldr
            _check_apart(y, "y", ((x, "x"), (w, "w"), (bias, "bias"), (None if same else residual, "residual")))

        def body():
            out = given if given is not None else self._torch.empty((t, n_out), dtype=x.dtype, device=dev)
            kept, keep = self._keep(save, t, n_out, x.dtype)
            work, size, at = self._forward_work(0, t, n_in, n_out, (x, ldx), (w, ldw))
            check(self._fn.dbs_linear(
                self._h, dt, t, n_in, n_out, x.data_ptr(), ldx, w.data_ptr(), ldw,
                None if bias is None else bias.data_ptr(), act_code, None if residual is None else residual.data_ptr(),
                ldr, out.data_ptr(), n_out if given is None else ldy, None if keep is None else ctypes.byref(keep), at, size))
            return out, kept
        out, kept = self._call(body, (x, w, bias, residual, given))
        if x.requires_grad or w.requires_grad or bias is not None and bias.requires_grad or \
                residual is not None and residual.requires_grad:
            out, kept = _no_graph(self._torch, "linear", (x, w, bias, residual), (out, kept))
        out = out[0] if one else out
        return out if save == "none" else (out, kept)

    def gated(self, x, w_gate, w_up, act="silu", save="none", h=None):
        """h = act(x w_gate^T) * (x w_up^T) for x [tokens, n_in] (or one token
        [n_in]); h may be preallocated.  With save "full" or "8bit" returns
        (h, gate, up): the projections as tensors or Checkpoints for
        ``gated_backward``."""
        act_code, save = _choice(act, ACTS, "act"), _choice(save, SAVES, "save")
        dt, dev = _dtype_code(self._torch, x, "x"), self.device
        one = x.dim() == 1
        if one:
            x = x.unsqueeze(0)
            h = None if h is None else h.unsqueeze(0)
        ldx = check_rows(x, "x", x.dtype, dev, None, None)
        t, n_in = x.shape
        ldg = check_rows(w_gate, "w_gate", x.dtype, dev, None, n_in)
        n_out = w_gate.shape[0]
        ldu = check_rows(w_up, "w_up", x.dtype, dev, n_out, n_in)
        given = h
        if h is not None:
            ldh = check_rows(h, "h", x.dtype, dev, t, n_out)
            _check_apart(h, "h", ((x, "x"), (w_gate, "w_gate"), (w_up, "w_up")))

        def body():
            out = given if given is not None else self._torch.empty((t, n_out), dtype=x.dtype, device=dev)
            gate, kg = self._keep(save, t, n_out, x.dtype)
            up, ku = self._keep(save, t, n_out, x.dtype)
            work, size, at = self._forward_work(1, t, n_in, n_out, (x, ldx), (w_gate, ldg), (w_up, ldu))
            check(self._fn.dbs_gated(
                self._h, dt, t, n_in, n_out, x.data_ptr(), ldx, w_gate.data_ptr(), ldg, w_up.data_ptr(), ldu, act_code,
                out.data_ptr(), n_out if given is None else ldh, None if kg is None else ctypes.byref(kg),
                None if ku is None else ctypes.byref(ku), at, size))
            return out, gate, up
        out, gate, up = self._call(body, (x, w_gate, w_up, given))
        if x.requires_grad or w_gate.requires_grad or w_up.requires_grad:
            out, gate, up = _no_graph(self._torch, "gated", (x, w_gate, w_up), (out, gate, up))
        out = out[0] if one else out
        return out if save == "none" else (out, gate, up)

    # -- backward
    def _work(self, gated, act, t, n_in, n_out, x_codes, want_db, *inputs):
        n = ctypes.c_size_t()
        whole = n_in % 8 == 0 and all(_whole(v, ld) for v, ld in inputs)
        check(self._fn.dbs_backward_work(self._h, gated, act, t, n_in, n_out, x_codes, want_db, whole, ctypes.byref(n)))
        return self._torch.empty(n.value, dtype=self._torch.uint8, device=self.device) if n.value else None, n.value

    def linear_backward(self, dy, x, w, pre=None, act="none", bias=False, need_dx=True, need_dw=True):
        """Gradients of ``linear``: (dx, dw, db) from dy [tokens, n_out], the
        layer's x and the saved pre (tensors or Checkpoints; pre only with an
        activation).  db is None without `bias`, dx and dw without their
        `need_`; the residual's gradient is dy."""
        torch, dev = self._torch, self.device
        act_code = _choice(act, ACTS, "act")
        dt = _dtype_code(torch, dy, "dy")
        ldy = check_rows(dy, "dy", dy.dtype, dev, None, None)
        t, n_out = dy.shape
        ldw = check_rows(w, "w", dy.dtype, dev, n_out, None)
        n_in = w.shape[1]
        hx, x_codes = self._held(x, "x", dy.dtype, t, n_in) if need_dw else (None, False)
        hp = self._held(pre, "pre", dy.dtype, t, n_out)[0] if act != "none" else None

        def body():
            dx = torch.empty((t, n_in), dtype=dy.dtype, device=dev) if need_dx else None
            dw = torch.empty((n_out, n_in), dtype=dy.dtype, device=dev) if need_dw else None
            db = torch.empty((n_out,), dtype=dy.dtype, device=dev) if bias else None
            work, size = self._work(0, act_code, t, n_in, n_out, x_codes, 1 if bias else 0, (dy, ldy), (w, ldw),
                                    *(((x, hx.ld),) if need_dw and not x_codes else ()))
            check(self._fn.dbs_linear_backward(
                self._h, dt, t, n_in, n_out, dy.data_ptr(), ldy, None if hx is None else ctypes.byref(hx), w.data_ptr(),
                ldw, None if hp is None else ctypes.byref(hp), act_code, None if dx is None else dx.data_ptr(), n_in,
                None if dw is None else dw.data_ptr(), n_in, None if db is None else db.data_ptr(),
                None if work is None else work.data_ptr(), size))
            return dx, dw, db
        return self._call(body, (dy, x if need_dw else None, w, pre if act != "none" else None))

    def gated_backward(self, dh, x, w_gate, w_up, gate, up, act="silu", need_dx=True, need_dw=True):
        """Gradients of ``gated``: (dx, dw_gate, dw_up) from dh [tokens, n_out],
        the layer's x and the saved gate and up (tensors or Checkpoints)."""
        torch, dev = self._torch, self.device
        act_code = _choice(act, ACTS, "act")
        dt = _dtype_code(torch, dh, "dh")
        ldh = check_rows(dh, "dh", dh.dtype, dev, None, None)
        t, n_out = dh.shape
        ldg = check_rows(w_gate, "w_gate", dh.dtype, dev, n_out, None)
        n_in = w_gate.shape[1]
        ldu = check_rows(w_up, "w_up", dh.dtype, dev, n_out, n_in)
        hx, x_codes = self._held(x, "x", dh.dtype, t, n_in) if need_dw else (None, False)
        hg, hu = self._held(gate, "gate", dh.dtype, t, n_out)[0], self._held(up, "up", dh.dtype, t, n_out)[0]

        def body():
            dx = torch.empty((t, n_in), dtype=dh.dtype, device=dev) if need_dx else None
            dwg = torch.empty((n_out, n_in), dtype=dh.dtype, device=dev) if need_dw else None
            dwu = torch.empty((n_out, n_in), dtype=dh.dtype, device=dev) if need_dw else None
            work, size = self._work(1, act_code, t, n_in, n_out, x_codes, 0, (w_gate, ldg), (w_up, ldu),
                                    *(((x, hx.ld),) if need_dw and not x_codes else ()))
            check(self._fn.dbs_gated_backward(
                self._h, dt, t, n_in, n_out, dh.data_ptr(), ldh, None if hx is None else ctypes.byref(hx),
                w_gate.data_ptr(), ldg, w_up.data_ptr(), ldu, ctypes.byref(hg), ctypes.byref(hu), act_code,
                None if dx is None else dx.data_ptr(), n_in, None if dwg is None else dwg.data_ptr(), n_in,
                None if dwu is None else dwu.data_ptr(), n_in, None if work is None else work.data_ptr(), size))
            return dx, dwg, dwu
        return self._call(body, (dh, x if need_dw else None, w_gate, w_up, gate, up))

    # -- checkpoints
    def pack(self, x):
        """x [rows, cols] (float16 or bfloat16) as a Checkpoint."""
        dt = _dtype_code(self._torch, x, "x")
        ld = check_rows(x, "x", x.dtype, self.device, None, None)
        rows, cols = x.shape

        def body():
            c = self._new_checkpoint(rows, cols, x.dtype)
            check(self._fn.dbs_pack(self._h, dt, rows, cols, x.data_ptr(), ld, c.codes.data_ptr(), c.exponents.data_ptr()))
            return c
        return self._call(body, (x,))

    def unpack(self, c, y=None):
        """The values of a Checkpoint [rows, cols], in its type."""
        torch = self._torch
        if not isinstance(c, Checkpoint):
            raise _arg_error("unpack takes a Checkpoint")
        if c.codes.dim() != 2:
            raise _arg_error(f"the codes of c must have 2 dimensions, not {c.codes.dim()}")
        if c.dtype not in (torch.float16, torch.bfloat16):
            raise _arg_error(f"c holds values of {c.dtype}, expected torch.float16 or torch.bfloat16")
        rows, cols = c.codes.shape
        check_checkpoint(torch, c, "c", c.dtype, self.device, rows, cols)
        ld = cols if y is None else check_rows(y, "y", c.dtype, self.device, rows, cols)
        if y is not None:
            _check_apart(y, "y", ((c.codes, "the codes of c"), (c.exponents, "the exponents of c")))

        def body():
            out = torch.empty((rows, cols), dtype=c.dtype, device=self.device) if y is None else y
            check(self._fn.dbs_unpack(self._h, DBS_BF16 if c.dtype == torch.bfloat16 else DBS_F16, rows, cols,
                                      c.codes.data_ptr(), c.exponents.data_ptr(), out.data_ptr(), ld))
            return out
        return self._call(body, (c, y))
