"""The edges of a feed-forward block on the MI355X -- Python binding.

The norm before a block, the join with the residual stream after it, dropout,
and their gradients (``include/dbspmspv.h``).  Argument marshalling only.

    before, after = Norm(w, eps=1e-6), Norm(g, b, kind="layer", eps=1e-5)
    h = ctx.norm(x, before)
    x, h = ctx.join(branch, x, after=after, before=before, gate=gate, p=0.1, rng=(seed, step))
    d = ctx.join_backward(dx, dh, branch, x, after=after, before=before, gate=gate, p=0.1, rng=(seed, step))
    dx, dw, db = ctx.norm_backward(dh, x, before, add=d.residual)
"""
from __future__ import annotations

import collections
import ctypes
import math
import operator

from . import _lib
from ._lib import check
from .layer_args import _arg_error, _check_apart, _choice, _dtype_code, _no_graph, check_rows, check_vector

NORMS = {"rms": _lib.DBS_NORM_RMS, "layer": _lib.DBS_NORM_LAYER}


class Norm:
    """A norm by rows: xh * weight + bias, with xh = x / sqrt(mean(x^2) + eps)
    ("rms") or (x - mean) / sqrt(var + eps) ("layer").  weight and bias are
    vectors of the call's type, or None (ones, zeros)."""

    __slots__ = ("weight", "bias", "kind", "eps")

    def __init__(self, weight=None, bias=None, kind="rms", eps=1e-6):
        self.weight, self.bias, self.kind, self.eps = weight, bias, kind, eps


JoinGrads = collections.namedtuple("JoinGrads", ["residual", "branch", "gate", "after_weight", "after_bias", "before_weight",
                                                 "before_bias"])


def _norm_desc(norm, name, dtype, device, n):
    """dbs_norm_desc of a Norm, or None."""
    if norm is None:
        return None
    if not isinstance(norm, Norm):
        raise _arg_error(f"{name} is a {type(norm).__name__}, expected a Norm")
    kind = _choice(norm.kind, NORMS, f"the kind of {name}")
    if not (0.0 <= norm.eps < math.inf):
        raise _arg_error(f"the eps of {name} is {norm.eps}, expected a finite number, at least 0")
    w, b = norm.weight, norm.bias
    if w is not None:
        check_vector(w, f"the weight of {name}", dtype, device, n)
    if b is not None:
        check_vector(b, f"the bias of {name}", dtype, device, n)
    return _lib.NormDesc(kind, norm.eps, None if w is None else w.data_ptr(), None if b is None else b.data_ptr())


def _params(norm):
    return (None, None) if norm is None else (norm.weight, norm.bias)


def _drop_desc(torch, p, rng, device):
    """(dbs_drop_desc or None, the tensor it reads or None)."""
    if not (0.0 <= p <= 1.0):
        raise _arg_error(f"p is {p}, expected a number from 0 to 1")
    if p == 0.0:
        return None, None
    if rng is None:
        raise _arg_error("dropout needs rng: (seed, offset), or an int64 tensor of the two")
    if isinstance(rng, torch.Tensor):
        check_vector(rng, "rng", torch.int64, device, 2)
        return _lib.DropDesc(p, 0, 0, rng.data_ptr()), rng
    try:
        seed, offset = (operator.index(v) for v in rng)
    except (TypeError, ValueError):
        raise _arg_error(f"rng is {rng!r}, expected (seed, offset), or an int64 tensor of the two") from None
    if not (0 <= seed < 1 << 64 and 0 <= offset < 1 << 64):
        raise _arg_error("seed and offset are whole numbers of 64 bits, not negative")
    return _lib.DropDesc(p, seed, offset, None), None


def _wants(tensors):
    for t in tensors:
        if t is not None and t.requires_grad:
            return True
    return False


def _at(t):
    return None if t is None else t.data_ptr()


def _ref(d):
    return None if d is None else ctypes.byref(d)


class EdgeOps:
    """Norms, joins and dropout of a LayerContext."""

    def _gate(self, gate, dtype, rows, n):
        """The elements from row to row of a gate: 0 for a vector."""
        if gate is None:
            return 0
        if gate.dim() == 1:
            check_vector(gate, "gate", dtype, self.device, n)
            return 0
        return max(1, check_rows(gate, "gate", dtype, self.device, rows, n))

    def norm(self, x, norm, to8=False, y=None):
        """norm(x) for x [tokens, n] (or one token [n]); y may be preallocated,
        also as x itself.  With to8 the result comes as row blocks of 8 bits
        (``Blocks8``) for ``linear8``: those of the 16-bit result."""
        torch, dev = self._torch, self.device
        dt = _dtype_code(torch, x, "x")
        one = x.dim() == 1
        if one:
            x = x.unsqueeze(0)
            y = None if y is None else y.unsqueeze(0)
        ldx = check_rows(x, "x", x.dtype, dev, None, None)
        t, n = x.shape
        if norm is None:
            raise _arg_error("norm is required")
        desc = _norm_desc(norm, "norm", x.dtype, dev, n)
        given = y
        if y is not None:
            if to8:
                raise _arg_error("y is a 16-bit result: not with to8")
            ldy = check_rows(y, "y", x.dtype, dev, t, n)
            same = y.data_ptr() == x.data_ptr() and ldy == ldx
            _check_apart(y, "y", ((None if same else x, "x"), (norm.weight, "weight"), (norm.bias, "bias")))

        def body():
            if to8:
                out = self._new_blocks(t, n, "row", x.dtype)
                check(self._fn.dbs_norm(self._h, dt, t, n, x.data_ptr(), ldx, ctypes.byref(desc), None, 0, out._ref()))
                return out
            out = given if given is not None else x.new_empty((t, n))
            check(self._fn.dbs_norm(self._h, dt, t, n, x.data_ptr(), ldx, ctypes.byref(desc), out.data_ptr(),
                                    n if given is None else ldy, None))
            return out
        out = self._call(body, (x, norm.weight, norm.bias, given))
        inputs = (x, norm.weight, norm.bias)
        if _wants(inputs):
            if to8:
                out.codes, = _no_graph(torch, "norm", inputs, (out.codes,))
            else:
                out, = _no_graph(torch, "norm", inputs, (out,))
        return out[0] if one and not to8 else out

    def _edge_work(self, rows, n, sums):
        size = ctypes.c_size_t()
        check(self._fn.dbs_edge_work(self._h, rows, n, sums, ctypes.byref(size)))
        if not size.value:
            return None, 0, None
        work = self._torch.empty(size.value, dtype=self._torch.uint8, device=self.device)
        return work, size.value, work.data_ptr()

    def norm_backward(self, dy, x, norm, add=None, need_dx=True, need_dw=True):
        """Gradients of ``norm`` at x: (dx, dweight, dbias) from dy [tokens, n];
        add [tokens, n] (a gradient that comes to x by another way) is added to dx.
        None for what the norm does not have or is not needed."""
        torch, dev = self._torch, self.device
        dt = _dtype_code(torch, dy, "dy")
        lddy = check_rows(dy, "dy", dy.dtype, dev, None, None)
        t, n = dy.shape
        ldx = check_rows(x, "x", dy.dtype, dev, t, n)
        if norm is None:
            raise _arg_error("norm is required")
        desc = _norm_desc(norm, "norm", dy.dtype, dev, n)
        ldadd = 0 if add is None else check_rows(add, "add", dy.dtype, dev, t, n)

        def body():
            new = lambda *shape: dy.new_empty(shape)  # noqa: E731
            dx = new(t, n) if need_dx else None
            dw = new(n) if need_dw and norm.weight is not None else None
            db = new(n) if need_dw and norm.bias is not None else None
            work, size, at = self._edge_work(t, n, (dw is not None) + (db is not None))
            check(self._fn.dbs_norm_backward(self._h, dt, t, n, dy.data_ptr(), lddy, x.data_ptr(), ldx, ctypes.byref(desc),
                                             _at(add), ldadd, _at(dx), n, _at(dw), _at(db), at, size))
            return dx, dw, db
        return self._call(body, (dy, x, norm.weight, norm.bias, add))

    def join(self, branch, residual, after=None, before=None, gate=None, scale=1.0, p=0.0, rng=None, to8=False, stream=None):
        """(stream, h): stream = scale * residual + gate * dropout(after(branch)) and
        h = before(stream) for branch and residual [tokens, n] (or one token [n]).

        after, before: ``Norm`` or None (h is None without before).  gate: a vector
        [n], or [tokens, n], or None.  Dropout with probability p takes rng, (seed,
        offset) or an int64 tensor of the two on the device, which a captured call
        reads anew; the backward pass takes the same.  stream may be preallocated,
        also as the residual itself.  With to8 h comes as row blocks of 8 bits."""
        torch, dev = self._torch, self.device
        dt = _dtype_code(torch, branch, "branch")
        one = branch.dim() == 1
        if one:
            branch = branch.unsqueeze(0)
            residual = None if residual is None else residual.unsqueeze(0)
            stream = None if stream is None else stream.unsqueeze(0)
        ldb = check_rows(branch, "branch", branch.dtype, dev, None, None)
        t, n = branch.shape
        dtype = branch.dtype
        ldr = check_rows(residual, "residual", dtype, dev, t, n)
        da, db = _norm_desc(after, "after", dtype, dev, n), _norm_desc(before, "before", dtype, dev, n)
        ldg = self._gate(gate, dtype, t, n)
        drop, rng_t = _drop_desc(torch, p, rng, dev)
        if to8 and before is None:
            raise _arg_error("to8 is of h, which needs a norm before")
        inputs = (branch, residual, *_params(after), *_params(before), gate)
        given = stream
        if stream is not None:
            lds = check_rows(stream, "stream", dtype, dev, t, n)
            same = stream.data_ptr() == residual.data_ptr() and lds == ldr
            names = ("branch", "residual", "after's weight", "after's bias", "before's weight", "before's bias", "gate")
            _check_apart(stream, "stream", tuple((None if same and v is residual else v, k) for v, k in zip(inputs, names)))

        def body():
            out = given if given is not None else branch.new_empty((t, n))
            h = h8 = None
            if to8:
                h8 = self._new_blocks(t, n, "row", dtype)
            elif before is not None:
                h = branch.new_empty((t, n))
            check(self._fn.dbs_join(self._h, dt, t, n, branch.data_ptr(), ldb, residual.data_ptr(), ldr, _ref(da), _ref(db),
                                    _at(gate), ldg, scale, _ref(drop), out.data_ptr(), n if given is None else lds, _at(h), n,
                                    None if h8 is None else h8._ref()))
            return out, h8 if to8 else h
        out, h = self._call(body, (*inputs, rng_t, given))
        if _wants(inputs):
            out, marked = _no_graph(torch, "join", inputs, (out, h.codes if to8 else h))
            if to8:
                h.codes = marked
            else:
                h = marked
        if one:
            out, h = out[0], h if to8 or h is None else h[0]
        return out, h

    def join_backward(self, dstream, dh, branch, stream, after=None, before=None, gate=None, scale=1.0, p=0.0, rng=None,
                      need_dw=True):
        """Gradients of ``join`` as JoinGrads (residual, branch, gate, after_weight,
        after_bias, before_weight, before_bias), None for what is not there or,
        without need_dw, the norms' and the gate's.

        dstream [tokens, n] may be None with a norm before; dh is the gradient of
        its result.  branch is needed with a gate or a norm after, stream (the
        output of ``join``) with a norm before."""
        torch, dev = self._torch, self.device
        lead = dstream if dstream is not None else dh
        dt = _dtype_code(torch, lead, "dstream")
        dtype = lead.dtype
        check_rows(lead, "dstream" if dstream is not None else "dh", dtype, dev, None, None)
        t, n = lead.shape
        if (dh is None) != (before is None):
            raise _arg_error("dh and before are given together")
        rows = lambda v, name: 0 if v is None else check_rows(v, name, dtype, dev, t, n)  # noqa: E731
        da, db = _norm_desc(after, "after", dtype, dev, n), _norm_desc(before, "before", dtype, dev, n)
        ldds, lddh = rows(dstream, "dstream"), rows(dh, "dh")
        ldg = self._gate(gate, dtype, t, n)
        if branch is None and (after is not None or gate is not None):
            raise _arg_error("branch is required with a norm after or a gate")
        if stream is None and before is not None:
            raise _arg_error("stream is required with a norm before")
        ldb, lds = rows(branch, "branch"), rows(stream, "stream")
        drop, rng_t = _drop_desc(torch, p, rng, dev)

        def body():
            new = lambda *shape: lead.new_empty(shape)  # noqa: E731
            vector = lambda v: new(n) if need_dw and v is not None else None  # noqa: E731
            wa, ba, wb, bb = (vector(v) for v in (*_params(after), *_params(before)))
            dgate = None if gate is None or not need_dw else new(n) if ldg == 0 else new(t, n)
            dres, dbranch = new(t, n), new(t, n)
            sums = sum(v is not None for v in (wa, ba, wb, bb)) + (dgate is not None and ldg == 0)
            work, size, at = self._edge_work(t, n, sums)
            check(self._fn.dbs_join_backward(
                self._h, dt, t, n, _at(dstream), ldds, _at(dh), lddh, _at(branch), ldb, _at(stream), lds, _ref(da), _ref(db),
                _at(gate), ldg, scale, _ref(drop), dres.data_ptr(), n, dbranch.data_ptr(), n, _at(dgate), n, _at(wa), _at(ba),
                _at(wb), _at(bb), at, size))
            return JoinGrads(dres, dbranch, dgate, wa, ba, wb, bb)
        return self._call(body, (dstream, dh, branch, stream, *_params(after), *_params(before), gate, rng_t))

    def dropout(self, x, p, rng, y=None):
        """x [tokens, n] (or one token [n]) with elements dropped with probability p
        (to the nearest 1/65536) and the others multiplied by 1 / (1 - p).  The
        choice is a function of rng and an element's place, so the same call on a
        gradient is the backward pass.  y may be preallocated, also as x itself."""
        torch, dev = self._torch, self.device
        dt = _dtype_code(torch, x, "x")
        one = x.dim() == 1
        if one:
            x = x.unsqueeze(0)
            y = None if y is None else y.unsqueeze(0)
        ldx = check_rows(x, "x", x.dtype, dev, None, None)
        t, n = x.shape
        drop, rng_t = _drop_desc(torch, p, rng, dev)
        drop = _lib.DropDesc(0.0, 0, 0, None) if drop is None else drop
        given = y
        if y is not None:
            ldy = check_rows(y, "y", x.dtype, dev, t, n)
            _check_apart(y, "y", ((None if y.data_ptr() == x.data_ptr() and ldy == ldx else x, "x"),))

        def body():
            out = given if given is not None else x.new_empty((t, n))
            check(self._fn.dbs_dropout(self._h, dt, t, n, x.data_ptr(), ldx, ctypes.byref(drop), out.data_ptr(),
                                       n if given is None else ldy))
            return out
        out = self._call(body, (x, rng_t, given))
        if x.requires_grad:
            out, = _no_graph(torch, "dropout", (x,), (out,), "its gradient is the same call on the gradient")
        return out[0] if one else out
