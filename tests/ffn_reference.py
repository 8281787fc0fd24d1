"""The feed-forward operators' definitions in 64 bits, each with a bound on what
32-bit sums and one rounding to the output's type may be off by."""
import math

import torch

# half a step, relative: finfo(t).eps / 2
HALF = {t: torch.finfo(t).eps / 2 for t in (torch.bfloat16, torch.float16, torch.float32)}
# half the distance of the smallest values (a result below the type's normal range is off by that)
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}
U = 2.0 ** -24


def within(got, want, bound, what):
    """|got - want| <= bound, elementwise; NaN only where `want` has one."""
    got = got.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    bad = ((got - want).abs() > bound) & ~torch.isnan(want)
    if bad.any():
        i = tuple(bad.nonzero()[0].tolist())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} out of bound; at {i} {got[i]} for {want[i]}, bound {bound[i]}")


def rounded(want, err, dtype):
    """A bound for a value within `err` of want and then rounded to dtype."""
    return err + HALF[dtype] * (want.abs() + err) + TINY[dtype]


def activation(g, act):
    """(act(g), act'(g)) in 64 bits; act 0 is SiLU, 1 GELU's tanh form."""
    if act == 0:
        s = torch.sigmoid(g)
        return g * s, s + g * s * (1 - s)
    k = math.sqrt(2 / math.pi)
    t = torch.tanh(k * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * k * (1 + 3 * 0.044715 * g * g)


def product(x, w, extra=0):
    """x w^T in 64 bits and the bound of an fp32 sum of its dim products in any
    order: each of the at most dim + extra additions rounds a partial sum of at
    most sum |x w| (an MFMA truncates, a whole step: 2 U)."""
    x, w = x.double(), w.double()
    return x @ w.t(), (x.shape[1] + extra + 1) * 2 * U * (x.abs() @ w.abs().t())


def gated(x, gate_w, up_w, gate_b, up_b, act, slack=0.0):
    """(y, bound before y's rounding, g, its bound, u, its bound).  slack: a
    further relative error of sum |x w| per product sum."""
    out = []
    for w, b in ((gate_w, gate_b), (up_w, up_b)):
        v, e = product(x, w, 2)
        e = e + slack * (x.double().abs() @ w.double().abs().t())
        if b is not None:
            v, e = v + b.double(), e + 2 * U * b.double().abs()
        out += [v, e + 2 * U * v.abs()]
    g, eg, u, eu = out
    a, _ = activation(g, act)
    # |act'| is at most 1.13; the sigmoid's argument and value are off by a few units of |g| U
    ea = 1.13 * eg + 16 * U * g.abs() * (1 + g.abs().clamp(max=100.0) * 0.3) + 4 * U * a.abs()
    return a * u, ea * u.abs() + a.abs() * eu + ea * eu + 2 * U * (a * u).abs(), g, eg, u, eu


def gated_bwd(x, gate_w, up_w, pre, dy, act, dtype):
    """The gradients and their bounds, given the stored g and u: dg and du carry
    one rounding to dtype into the products."""
    F = gate_w.shape[0]
    g, u, d = pre[:, :F].double(), pre[:, F:].double(), dy.double()
    a, slope = activation(g, act)
    dg, du = d * u * slope, d * a
    small = 32 * U * (1 + g.abs().clamp(max=100.0))
    eg, eu = (d * u).abs() * small * 1.13, d.abs() * g.abs().clamp(min=1e-30) * small
    rg, ru = rounded(dg, eg, dtype), rounded(du, eu, dtype)
    x, wg, wu = x.double(), gate_w.double(), up_w.double()
    r = {}
    dx = dg @ wg + du @ wu
    mag = (dg.abs() + rg) @ wg.abs() + (du.abs() + ru) @ wu.abs()
    r["dx"] = dx, rg @ wg.abs() + ru @ wu.abs() + (2 * F + 4) * 2 * U * mag
    M = x.shape[0]
    for name, v, e in (("gate", dg, rg), ("up", du, ru)):
        r[f"d{name}_w"] = v.t() @ x, e.t() @ x.abs() + (M + 4) * 2 * U * ((v.abs() + e).t() @ x.abs())
    for name, v, e in (("gate", dg, eg), ("up", du, eu)):
        r[f"d{name}_b"] = v.sum(0), e.sum(0) + (M + 4) * U * (v.abs() + e).sum(0)
    return r


def lora(x, w, bias, a, b, scale, ids, dtype):
    """(y, bound before its rounding) for ids >= -1; rows below -1 are zeros."""
    y, e = product(x, w, 4)
    n = a.shape[0]
    if bias is not None:
        y, e = y + bias.double(), e + 4 * U * bias.double().abs()
    two = HALF[dtype] ** 2 * 2      # what the rounding and the rounded remainder leave
    for i in range(n):
        rows = (ids == i).nonzero()[:, 0]
        if len(rows) == 0:
            continue
        s = float(scale[i])
        t, et = product(x[rows], a[i], 2)
        t, et = t * s, (et + 2 * U * t.abs()) * abs(s)
        et = et + two * t.abs() + TINY[dtype]
        bb = b[i].double()
        y[rows] += t @ bb.t()
        e[rows] += et @ bb.abs().t() + (2 * a.shape[1] + 4) * 2 * U * ((t.abs() + et) @ bb.abs().t())
    e = e + 2 * U * y.abs()
    y[ids >= n] = float("nan")
    y[ids < -1] = 0
    return y, e


def rmsnorm(x, resid, gamma, eps):
    """(s, y, relative bound of y before its rounding)"""
    s = x.double() + resid.double() if resid is not None else x.double()
    q = 1 / torch.sqrt((s * s).mean(1, keepdim=True) + eps)
    y = s * q
    if gamma is not None:
        y = y * gamma.double()
    # the sum of squares takes dim / 64 additions a lane and a few more, each of its fp32 terms two roundings
    return s, y, (s.shape[1] / 64 + 24) * U


def rmsnorm_bwd(s, dy, dsum, gamma, eps):
    """{name: (value, bound)}"""
    s, dy = s.double(), dy.double()
    D = s.shape[1]
    q = 1 / torch.sqrt((s * s).mean(1, keepdim=True) + eps)
    n, g = s * q, dy * gamma.double() if gamma is not None else dy
    along = (g * n).mean(1, keepdim=True)
    dx = q * (g - n * along)
    rel = (D / 64 + 32) * U
    e = rel * q * (g.abs() + n.abs() * ((g * n).abs().mean(1, keepdim=True) + along.abs()))
    if dsum is not None:
        dx = dx + dsum.double()
        e = e + U * dsum.double().abs()
    M = s.shape[0]
    dgamma = (dy * n).sum(0)
    # a workgroup's rows (all of them where one wave takes them), then up to 1024 parts in 16 sums
    return {"dx": (dx, e + U * dx.abs()), "dgamma": (dgamma, (M / 4 + 100) * U * (dy * n).abs().sum(0) + rel * (dy * n).abs().sum(0))}


def e4m3_steps(v):
    """Half the distance of e4m3 values around v."""
    return torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 4)
