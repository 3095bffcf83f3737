"""Norms, joins and dropout in 64 bits, with bounds on what the kernels may
differ from them by.

Values go through the formulas as pairs (value, bound of its error).  With u =
2^-24 a sum in 32 bits of n terms is off by at most d u times the sum of their
magnitudes, d the number of terms added in a row: a lane of the kernels adds at
most n / 64 of a row's, then the lanes and waves are added, d = n / 64 + 64; sums
over t rows: d = t + 64.  Every other operation is off by u of its result, the
root and the division by less than 2^-22 together.  What is rounded to 16 bits is
off by half a step of the type at the end."""
import numpy as np
import torch

from layer_ref import rounded

U32 = 2.0 ** -24
MASK = 0xFFFFFFFF


def philox(counter, key):
    """Philox4x32-10: four words from four words and a key of two (Salmon et al., 2011)."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [b >> 32 ^ c[1] ^ k[0], b & MASK, a >> 32 ^ c[3] ^ k[1], a & MASK]
        k = [(k[0] + 0x9E3779B9) & MASK, (k[1] + 0xBB67AE85) & MASK]
    return c


def threshold(p):
    return int(np.floor(p * 65536 + 0.5))


def factor(rows, n, p, rng, first=0):
    """What dropout multiplies each element by (of rows from `first` on)."""
    t = threshold(p)
    if t == 0:
        return torch.ones((rows, n), dtype=torch.float64)
    chunks = -(-n // 8)
    bits = np.zeros((rows, chunks * 8), np.int64)
    seed, offset = rng
    c = np.arange(first * chunks, (first + rows) * chunks, dtype=np.uint64)
    x = [c & np.uint64(MASK), c >> np.uint64(32), np.full_like(c, offset & MASK), np.full_like(c, offset >> 32)]
    k = [seed & MASK, seed >> 32]
    for _ in range(10):
        a, b = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        s = np.uint64(32)
        x = [(b >> s) ^ x[1] ^ np.uint64(k[0]), b & np.uint64(MASK), (a >> s) ^ x[3] ^ np.uint64(k[1]), a & np.uint64(MASK)]
        k = [(k[0] + 0x9E3779B9) & MASK, (k[1] + 0xBB67AE85) & MASK]
    for j in range(8):
        bits[:, j::8] = ((x[j // 2] >> np.uint64(16 * (j % 2))) & np.uint64(0xFFFF)).astype(np.int64).reshape(rows, chunks)
    keep = bits[:, :n] >= t
    return torch.from_numpy(keep).double() * (65536 / (65536 - t) if t < 65536 else 0.0)


class Row:
    """A norm of the rows of x (value, bound)."""

    def __init__(self, x, ex, norm):
        self.kind, n = norm.kind, x.shape[1]
        e = (n / 64 + 64) * U32
        self.w = torch.ones(n).double() if norm.weight is None else norm.weight.cpu().double()
        self.b = torch.zeros(n).double() if norm.bias is None else norm.bias.cpu().double()
        mean = lambda v: v.mean(1, keepdim=True)  # noqa: E731
        c, ec = x, ex
        if self.kind == "layer":
            c = x - mean(x)
            ec = ex + e * mean(x.abs()) + mean(ex) + U32 * c.abs()
        var = mean(c * c)
        evar = mean(2 * c.abs() * ec + ec * ec) + e * var
        root = (var + norm.eps).sqrt()
        self.rstd = 1 / root
        self.rel = torch.where(var + norm.eps > 0, evar / (var + norm.eps), torch.zeros_like(var)) + 2.0 ** -22
        self.xh = c * self.rstd
        self.exh = ec * self.rstd * (1 + self.rel) + self.xh.abs() * (self.rel + 2 * U32)
        self.e = e

    def out(self):
        y = self.xh * self.w + self.b
        return y, self.exh * self.w.abs() + 2 * U32 * (y.abs() + (self.xh * self.w).abs())

    def back(self, dy, edy):
        """((dx, bound), (dweight, bound), (dbias, bound))"""
        mean = lambda v: v.mean(1, keepdim=True)  # noqa: E731
        g = dy * self.w
        eg = edy * self.w.abs() + U32 * g.abs()
        m1 = mean(g * self.xh)
        em1 = mean(eg * self.xh.abs() + (g.abs() + eg) * self.exh) + self.e * mean((g * self.xh).abs())
        m2, em2 = torch.zeros_like(m1), torch.zeros_like(m1)
        if self.kind == "layer":
            m2 = mean(g)
            em2 = mean(eg) + self.e * mean(g.abs())
        inner = g - self.xh * m1 - m2
        ein = eg + self.exh * (m1.abs() + em1) + self.xh.abs() * em1 + em2
        ein = ein + 4 * U32 * (g.abs() + (self.xh * m1).abs() + m2.abs())
        dx = inner * self.rstd
        edx = ein * self.rstd * (1 + self.rel) + dx.abs() * (self.rel + 4 * U32)
        return (dx, edx), column(dy * self.xh, edy * self.xh.abs() + (dy.abs() + edy) * self.exh), column(dy, edy)


def column(v, ev):
    return v.sum(0), ev.sum(0) + (len(v) + 64) * U32 * v.abs().sum(0)


def _exact(v):
    v = v.cpu().double()
    return v, torch.zeros_like(v)


def norm(x, nm):
    dt = x.dtype
    y, ey = Row(*_exact(x), nm).out()
    return y, rounded(y, ey, dt)


def norm_backward(dy, x, nm, add=None):
    dt = dy.dtype
    (dx, edx), (dw, edw), (db, edb) = Row(*_exact(x), nm).back(*_exact(dy))
    if add is not None:
        dx = dx + add.cpu().double()
        edx = edx + U32 * dx.abs()
    out = {"dx": (dx, edx)}
    if nm.weight is not None:
        out["dweight"] = (dw, edw)
    if nm.bias is not None:
        out["dbias"] = (db, edb)
    return {k: (v, rounded(v, e, dt)) for k, (v, e) in out.items()}


def _branch(branch, after, p, rng):
    """dropout(after(branch)) with its parts."""
    b, eb = _exact(branch)
    row = None if after is None else Row(b, eb, after)
    u, eu = (b, eb) if row is None else row.out()
    f = factor(*b.shape, p, rng)
    return row, f, u * f, (eu + U32 * u.abs()) * f


def _gate(gate):
    return 1.0 if gate is None else gate.cpu().double()


def join(branch, residual, after, before, gate, scale, p, rng):
    dt = branch.dtype
    _, _, v, ev = _branch(branch, after, p, rng)
    g, r = _gate(gate), residual.cpu().double()
    scale = float(np.float32(scale))
    s = scale * r + g * v
    es = (g * ev).abs() + 2 * U32 * ((scale * r).abs() + (g * v).abs())
    out = {"stream": (s, rounded(s, es, dt))}
    if before is not None:
        h, eh = Row(s, es, before).out()
        out["h"] = (h, rounded(h, eh, dt))
    return out


def join_backward(dstream, dh, branch, stream, after, before, gate, scale, p, rng):
    lead = dstream if dstream is not None else dh
    dt = lead.dtype
    scale = float(np.float32(scale))
    d, ed = _exact(torch.zeros_like(lead) if dstream is None else dstream)
    out = {}
    if before is not None:
        (m, em), dw, db = Row(*_exact(stream), before).back(*_exact(dh))
        d, ed = d + m, em + U32 * (d + m).abs() + U32 * m.abs()
        if before.weight is not None:
            out["before_weight"] = dw
        if before.bias is not None:
            out["before_bias"] = db
    out["residual"] = d * scale, ed * abs(scale) + U32 * (d * scale).abs()
    g = _gate(gate)
    if branch is not None:
        row, f, v, ev = _branch(branch, after, p, rng)
    else:
        row, f = None, factor(*lead.shape, p, rng)
    if gate is not None:
        w, ew = d * v, ed * v.abs() + (d.abs() + ed) * ev + 2 * U32 * (d * v).abs()
        out["gate"] = (w, ew) if gate.dim() == 2 else column(w, ew)
    du, edu = d * g * f, (ed * f * (g if gate is None else g.abs())) + 3 * U32 * (d * g * f).abs()
    if row is not None:
        (du, edu), dw, db = row.back(du, edu)
        if after.weight is not None:
            out["after_weight"] = dw
        if after.bias is not None:
            out["after_bias"] = db
    out["branch"] = du, edu
    return {k: (v, rounded(v, e, dt)) for k, (v, e) in out.items()}
