"""The dense layer operators' definitions in 64 bits, with bounds on what the
kernels may differ from them by.

The bounds follow from the arithmetic.  With u half a unit in the last place
of the element type (bf16 2^-8, fp16 2^-11, and 2^-25 absolute where fp16 is
subnormal) a product of n terms summed in 32 bits in any order is off by at
most (n + 2) 2^-24 times the sum S of the terms' magnitudes; an activation
changes by at most 1.2 times its argument's error (the largest slope, of GELU,
is 1.13) and is itself evaluated to 2^-20 of its magnitude (its slope: 2^-20
absolute times the incoming gradient); every rounding to the element type adds
u of the result, and a rounded factor dz adds the rounding of each of its
terms."""
import torch

CK = 32
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
LEAST_EXP = {torch.bfloat16: -127, torch.float16: -24}
MAX = {torch.bfloat16: torch.finfo(torch.bfloat16).max, torch.float16: 65504.0}


def act(z, kind):
    if kind == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if kind == "silu":
        return z * torch.sigmoid(z)
    if kind == "gelu":
        return 0.5 * z * torch.erfc(-z / 2 ** 0.5)
    if kind == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh((2 / torch.pi) ** 0.5 * (z + 0.044715 * z ** 3)))
    return z


def slope(z, kind):
    if kind == "none":
        return torch.ones_like(z)
    if kind == "relu":
        return (z > 0).double()
    if kind == "silu":
        s = torch.sigmoid(z)
        return s + z * s * (1 - s)
    if kind == "gelu":
        return 0.5 * torch.erfc(-z / 2 ** 0.5) + z * torch.exp(-z * z / 2) / (2 * torch.pi) ** 0.5
    c = (2 / torch.pi) ** 0.5
    t = torch.tanh(c * (z + 0.044715 * z ** 3))
    return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)


def sum_err(n, s):
    return (n + 2) * 2.0 ** -24 * s


def rounded(v, err, dtype):
    return err + U[dtype] * (v.abs() + err) + TINY[dtype]


def linear(x, w, bias, kind, residual):
    """(y, bound of y, pre, bound of pre) for 16-bit tensors."""
    dt = x.dtype
    x, w = x.double(), w.double()
    z, ez = x @ w.T, sum_err(x.shape[1], x.abs() @ w.abs().T)
    if bias is not None:
        z = z + bias.double()
        ez = ez + 2.0 ** -24 * (z.abs() + ez)
    f = act(z, kind)
    y, ey = f, 1.2 * ez + 2.0 ** -20 * f.abs()
    if residual is not None:
        y = y + residual.double()
        ey = ey + 2.0 ** -24 * (y.abs() + ey)
    return y, rounded(y, ey, dt), z, rounded(z, ez, dt)


def gated(x, wg, wu, kind):
    """(h, bound, gate, bound, up, bound)."""
    dt = x.dtype
    x, wg, wu = x.double(), wg.double(), wu.double()
    n = x.shape[1]
    g, eg = x @ wg.T, sum_err(n, x.abs() @ wg.abs().T)
    u, eu = x @ wu.T, sum_err(n, x.abs() @ wu.abs().T)
    f = act(g, kind)
    ef = 1.2 * eg + 2.0 ** -20 * f.abs()
    h = f * u
    eh = ef * (u.abs() + eu) + f.abs() * eu + 2.0 ** -23 * h.abs()
    return h, rounded(h, eh, dt), g, rounded(g, eg, dt), u, rounded(u, eu, dt)


def linear_backward(dy, x, w, pre, kind):
    """{name: (gradient, bound)} of values in 64 bits (x, pre: the values that
    the backward pass sees)."""
    dt = dy.dtype
    dy, w = dy.double(), w.double()
    dz = dy if kind == "none" else dy * slope(pre, kind)
    raw = torch.zeros_like(dy) if kind == "none" else 2.0 ** -20 * dy.abs() + 2.0 ** -23 * dz.abs()
    e = raw if kind == "none" else rounded(dz, raw, dt)
    t, n_out = dy.shape
    dx, mx = dz @ w, (dz.abs() + e) @ w.abs()
    dw, mw = dz.T @ x, (dz.abs() + e).T @ x.abs()
    db = dz.sum(0)
    return {"dx": (dx, rounded(dx, e @ w.abs() + sum_err(n_out, mx), dt)),
            "dw": (dw, rounded(dw, e.T @ x.abs() + sum_err(t, mw), dt)),
            "db": (db, rounded(db, raw.sum(0) + sum_err(t, (dz.abs() + raw).sum(0)), dt))}


def gated_backward(dh, x, wg, wu, gate, up, kind):
    dt = dh.dtype
    dh, wg, wu = dh.double(), wg.double(), wu.double()
    f = act(gate, kind)
    dg, du = dh * up * slope(gate, kind), dh * f
    eg = rounded(dg, 2.0 ** -20 * (dh * up).abs() + 2.0 ** -22 * dg.abs(), dt)
    eu = rounded(du, 2.0 ** -20 * du.abs(), dt)
    t, n_out = dh.shape
    dx = dg @ wg + du @ wu
    mx = (dg.abs() + eg) @ wg.abs() + (du.abs() + eu) @ wu.abs()
    out = {"dx": (dx, rounded(dx, eg @ wg.abs() + eu @ wu.abs() + sum_err(2 * n_out, mx), dt))}
    for name, d, e in (("dw_gate", dg, eg), ("dw_up", du, eu)):
        dw = d.T @ x
        out[name] = (dw, rounded(dw, e.T @ x.abs() + sum_err(t, (d.abs() + e).T @ x.abs()), dt))
    return out


def pack(x):
    """(codes, exponents) of a 16-bit tensor on the CPU, group by group with
    exact arithmetic in 64 bits."""
    x64 = x.double()
    rows, cols = x.shape
    codes = torch.zeros((rows, cols), dtype=torch.int8)
    exps = torch.zeros((rows, -(-cols // CK)), dtype=torch.uint8)
    for k in range(exps.shape[1]):
        v = x64[:, k * CK:(k + 1) * CK]
        a = torch.where(v.isfinite(), v.abs(), 0.0).amax(1)
        e = torch.full((rows,), LEAST_EXP[x.dtype], dtype=torch.int64)
        for cand in range(LEAST_EXP[x.dtype], 130):
            e = torch.where(a > 127 * 2.0 ** cand, torch.full_like(e, cand + 1), e)
        c = torch.round(torch.nan_to_num(v, nan=0.0, posinf=0.0, neginf=0.0) * (2.0 ** -e.double())[:, None])
        codes[:, k * CK:(k + 1) * CK] = torch.where(v.isfinite(), c, -128.0).to(torch.int8)
        exps[:, k] = (e + 127).to(torch.uint8)
    return codes, exps


def unpack(codes, exps, dtype):
    e = (exps.double() - 127).repeat_interleave(CK, 1)[:, :codes.shape[1]]
    v = (codes.double() * 2.0 ** e).clamp(-MAX[dtype], MAX[dtype])
    return torch.where(codes == -128, float("nan"), v)


def check(got, want, bound, label):
    got = got.double()
    assert got.shape == want.shape, (label, got.shape, want.shape)
    nan = want.isnan()
    assert torch.equal(got.isnan(), nan), f"{label}: NaN in other places"
    inf = want.isinf()
    assert torch.equal(got[inf], want[inf]), f"{label}: infinities differ"
    ok = ~(nan | inf)
    over = (got[ok] - want[ok]).abs() - bound[ok]
    if over.numel() and not bool((over <= 0).all()):
        i = int(over.argmax())
        raise AssertionError(f"{label}: {int((over > 0).sum())} of {over.numel()} values off, worst {float(got[ok][i])} for "
                             f"{float(want[ok][i])} (may differ by {float(bound[ok][i])})")
