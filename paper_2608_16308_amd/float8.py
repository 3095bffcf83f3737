"""Products in 8-bit floating point on the MI355X -- Python binding.

Matrices in blocks of e4m3 codes with a power of two for each block of 128, and
the linear layer on them (``include/dbspmspv.h``).  Argument marshalling only.

    w8 = ctx.pack8(w, block="tile")                    # weights, laid out once
    y = ctx.linear8(x, w8, bias=bias, residual=r)      # x in 16 bits, or
    x8 = ctx.norm(x, norm, to8=True)                   # packed by what made it
    y = ctx.linear8(x8, w8)
    dx, dw, db = ctx.linear8_backward(dy, x8, w8, bias=True)
"""
from __future__ import annotations

import ctypes

from . import _lib
from ._lib import DBS_BF16, DBS_ERR_UNSUPPORTED, DBS_F16, DbsError, check
from .layer_args import (MAX_DIM, _arg_error, _check_apart, _choice, _dtype_code, _no_graph, _too_large, check_rows,
                         check_vector)

BLOCK8 = _lib.DBS_BLOCK8
BLOCKS = {"row": 0, "tile": 1}
MAX_SUM = 1 << 24  # elements of a product's sum
BY = "the products' gradients are those of LayerContext.linear8_backward"


def _up(n, by):
    return -(-n // by) * by


class Blocks8:
    """A matrix [rows, cols] in 8-bit floating point: ``codes`` float8_e4m3fn
    [rows, cols in whole blocks of 128] with zeros behind the last column,
    ``exponents`` uint8, one for each block of 128 columns of a row (block
    "row") or of 128 rows ("tile"), rows of them in whole fours (both contiguous
    device tensors); a value is code * 2^(exponent - 127).  ``dtype`` is the type
    of its values (float16 or bfloat16).  Where it was made of a tensor that requires
    a gradient, its codes do too: what autograd follows back to it raises."""

    __slots__ = ("codes", "exponents", "block", "shape", "dtype")

    def __init__(self, codes, exponents, block, shape, dtype):
        self.codes, self.exponents, self.block, self.shape, self.dtype = codes, exponents, block, tuple(shape), dtype

    @property
    def device(self):
        return self.codes.device

    @property
    def requires_grad(self):
        return self.codes.requires_grad

    def nbytes(self):
        return self.codes.numel() + self.exponents.numel()

    def _ref(self):
        return ctypes.byref(_lib.Blocks(self.codes.data_ptr(), self.exponents.data_ptr()))


def blocks_shapes(rows, cols, block):
    """Shapes of the codes and exponents of a matrix."""
    groups = -(-rows // BLOCK8) if block == "tile" else rows
    return (rows, _up(cols, BLOCK8)), (groups, _up(-(-cols // BLOCK8), 4))


def check_blocks(torch, c, name, dtype, device, rows, cols, block):
    """One matrix argument in blocks (None: any type or size)."""
    if len(c.shape) != 2 or min(c.shape) < 0:
        raise _arg_error(f"{name} has shape {c.shape}, expected two sizes")
    if max(c.shape) > MAX_DIM:
        raise _too_large(c.shape, name)
    if c.block != block:
        raise _arg_error(f"{name} is in {c.block!r} blocks, expected {block!r}")
    if dtype is not None and c.dtype != dtype:
        raise _arg_error(f"{name} holds values of {c.dtype}, expected {dtype}")
    if (rows is not None and c.shape[0] != rows) or (cols is not None and c.shape[1] != cols):
        raise _arg_error(f"{name} has shape {c.shape}, expected ({'any' if rows is None else rows}, "
                         f"{'any' if cols is None else cols})")
    codes, exps = blocks_shapes(*c.shape, block)
    for t, part, dt, shape, align in ((c.codes, "codes", torch.float8_e4m3fn, codes, 16),
                                      (c.exponents, "exponents", torch.uint8, exps, 4)):
        if t.device != device or t.dtype != dt or tuple(t.shape) != shape or not t.is_contiguous() or t.data_ptr() % align:
            raise _arg_error(f"the {part} of {name} must be a contiguous {dt} tensor {shape} on {device}, aligned to {align} "
                             f"bytes, not {t.dtype} {tuple(t.shape)} on {t.device}")


def _check_sum(n, name):
    if n > MAX_SUM:
        raise DbsError(DBS_ERR_UNSUPPORTED, f"{name} is {n}: a product's sum has at most 2^24 elements")


class Float8Ops:
    """Blocks of 8 bits and their products, of a LayerContext."""

    def _new_blocks(self, rows, cols, block, dtype):
        torch = self._torch
        codes, exps = blocks_shapes(rows, cols, block)
        return Blocks8(torch.empty(codes, dtype=torch.float8_e4m3fn, device=self.device),
                       torch.empty(exps, dtype=torch.uint8, device=self.device), block, (rows, cols), dtype)

    def pack8(self, x, block="row", across=False):
        """x [rows, cols] (float16 or bfloat16) as Blocks8: with an exponent for 128
        columns of a row ("row": activations) or of 128 rows ("tile": weights).
        across: the blocks of its transpose [cols, rows]."""
        torch = self._torch
        dt = _dtype_code(torch, x, "x")
        tile = _choice(block, BLOCKS, "block")
        ld = check_rows(x, "x", x.dtype, self.device, None, None)
        rows, cols = x.shape

        def body():
            out = self._new_blocks(*((cols, rows) if across else (rows, cols)), block, x.dtype)
            check(self._fn.dbs_pack8(self._h, dt, rows, cols, x.data_ptr(), ld, tile, 1 if across else 0, out._ref()))
            return out
        out = self._call(body, (x,))
        if x.requires_grad:
            out.codes, = _no_graph(torch, "pack8", (x,), (out.codes,), BY)
        return out

    def unpack8(self, c, y=None):
        """The values of a Blocks8 [rows, cols] in its type, limited to that type's
        largest finite number."""
        torch = self._torch
        if not isinstance(c, Blocks8):
            raise _arg_error("unpack8 takes a Blocks8")
        if c.dtype not in (torch.float16, torch.bfloat16):
            raise _arg_error(f"c holds values of {c.dtype}, expected torch.float16 or torch.bfloat16")
        tile = _choice(c.block, BLOCKS, "the block of c")
        check_blocks(torch, c, "c", c.dtype, self.device, None, None, c.block)
        rows, cols = c.shape
        ld = cols if y is None else check_rows(y, "y", c.dtype, self.device, rows, cols)
        if y is not None:
            _check_apart(y, "y", ((c.codes, "the codes of c"), (c.exponents, "the exponents of c")))

        def body():
            out = torch.empty((rows, cols), dtype=c.dtype, device=self.device) if y is None else y
            check(self._fn.dbs_unpack8(self._h, DBS_BF16 if c.dtype == torch.bfloat16 else DBS_F16, rows, cols, tile, c._ref(),
                                       out.data_ptr(), ld))
            return out
        out = self._call(body, (c, y))
        if c.requires_grad:
            out, = _no_graph(torch, "unpack8", (c.codes,), (out,), BY)
        return out

    def linear8(self, x, w, bias=None, residual=None, y=None):
        """y = x w^T + bias + residual with both factors in 8 bits: w Blocks8 [n_out,
        n_in] in "tile" blocks, x [tokens, n_in] Blocks8 in "row" blocks, or a 16-bit
        tensor (or one token [n_in]), which is brought into such blocks first.  y, in
        the type of x, may be preallocated, also as the residual."""
        torch, dev = self._torch, self.device
        if not isinstance(w, Blocks8):
            raise _arg_error("w must be a Blocks8 in tile blocks")
        held = isinstance(x, Blocks8)
        dt = _dtype_code(torch, x, "x")
        dtype = x.dtype
        one = not held and x.dim() == 1
        if one:
            x = x.unsqueeze(0)
            residual = None if residual is None else residual.unsqueeze(0)
            y = None if y is None else y.unsqueeze(0)
        if held:
            check_blocks(torch, x, "x", dtype, dev, None, None, "row")
        ldx = 0 if held else check_rows(x, "x", dtype, dev, None, None)
        t, n_in = x.shape
        _check_sum(n_in, "n_in")
        check_blocks(torch, w, "w", None, dev, None, n_in, "tile")
        n_out = w.shape[0]
        if bias is not None:
            check_vector(bias, "bias", dtype, dev, n_out)
        ldr = 0 if residual is None else check_rows(residual, "residual", dtype, dev, t, n_out)
        given = y
        if y is not None:
            ldy = check_rows(y, "y", dtype, dev, t, n_out)
            same = residual is not None and y.data_ptr() == residual.data_ptr() and ldy == ldr
            _check_apart(y, "y", ((x.codes if held else x, "x"), (x.exponents if held else None, "x"), (w.codes, "w"),
                                  (w.exponents, "w"), (bias, "bias"), (None if same else residual, "residual")))

        def body():
            out = given if given is not None else torch.empty((t, n_out), dtype=dtype, device=dev)
            work, size = None, 0
            if not held:
                need = ctypes.c_size_t()
                check(self._fn.dbs_linear8_work(self._h, t, n_in, n_out, ctypes.byref(need)))
                size = need.value
                work = torch.empty(size, dtype=torch.uint8, device=dev) if size else None
            check(self._fn.dbs_linear8(
                self._h, dt, t, n_in, n_out, None if held else x.data_ptr(), ldx, x._ref() if held else None, w._ref(),
                None if bias is None else bias.data_ptr(), None if residual is None else residual.data_ptr(), ldr,
                out.data_ptr(), n_out if given is None else ldy, None if work is None else work.data_ptr(), size))
            return out
        out = self._call(body, (x, w, bias, residual, given))
        if x.requires_grad or w.requires_grad or bias is not None and bias.requires_grad or \
                residual is not None and residual.requires_grad:
            out, = _no_graph(torch, "linear8", (x.codes if held else x, w.codes, bias, residual), (out,))
        return out[0] if one else out

    def linear8_backward(self, dy, x, w, bias=False, need_dx=True, need_dw=True):
        """Gradients of ``linear8``: (dx, dw, db) from dy [tokens, n_out], the layer's
        x (Blocks8 or a 16-bit tensor) and w, with dy (and for dw, in blocks of 128
        tokens, dy and x) brought into 8 bits.  db is None without `bias`, dx and dw
        without their `need_`; the residual's gradient is dy."""
        torch, dev = self._torch, self.device
        dt = _dtype_code(torch, dy, "dy")
        lddy = check_rows(dy, "dy", dy.dtype, dev, None, None)
        t, n_out = dy.shape
        _check_sum(t, "the number of tokens")
        _check_sum(n_out, "n_out")
        if not isinstance(w, Blocks8):
            raise _arg_error("w must be a Blocks8 in tile blocks")
        check_blocks(torch, w, "w", None, dev, n_out, None, "tile")
        n_in = w.shape[1]
        held, ldx = isinstance(x, Blocks8), 0
        if need_dw:
            if held:
                check_blocks(torch, x, "x", dy.dtype, dev, t, n_in, "row")
            else:
                ldx = check_rows(x, "x", dy.dtype, dev, t, n_in)

        def body():
            new = lambda *shape: torch.empty(shape, dtype=dy.dtype, device=dev)  # noqa: E731
            dx = new(t, n_in) if need_dx else None
            dw = new(n_out, n_in) if need_dw else None
            db = new(n_out) if bias else None
            need = ctypes.c_size_t()
            check(self._fn.dbs_linear8_backward_work(self._h, t, n_in, n_out, int(bool(need_dx)), int(bool(need_dw)),
                                                     int(bool(bias)), ctypes.byref(need)))
            work = torch.empty(need.value, dtype=torch.uint8, device=dev) if need.value else None
            check(self._fn.dbs_linear8_backward(
                self._h, dt, t, n_in, n_out, dy.data_ptr(), lddy, x.data_ptr() if need_dw and not held else None, ldx,
                x._ref() if need_dw and held else None, w._ref(), None if dx is None else dx.data_ptr(), n_in,
                None if dw is None else dw.data_ptr(), n_in, None if db is None else db.data_ptr(),
                None if work is None else work.data_ptr(), need.value))
            return dx, dw, db
        return self._call(body, (dy, x if need_dw else None, w))
