"""The cross-attention sub-block's operators' definitions in 64 bits, each with
a bound on what 32-bit sums and the roundings that include/xema_cross.h names may
be off by."""
import math

import torch

from ffn_reference import HALF, TINY, U, activation, product, rounded, within  # noqa: F401  (what the tests use)


def layernorm(x, resid, gamma, beta, eps):
    """(s, y, bound of y before its rounding)"""
    s = x.double() + resid.double() if resid is not None else x.double()
    D = s.shape[1]
    # a lane adds D / 64 terms, then a tree over lanes and waves; s itself is one rounding
    sums = (D / 64 + 14) * U
    em = (sums + U) * s.abs().mean(1, keepdim=True)
    e = s - s.mean(1, keepdim=True)
    var = (e * e).mean(1, keepdim=True)
    q = 1 / torch.sqrt(var + eps)
    n = e * q
    # s - mean: the mean's error and two roundings; 1 / sqrt(var + eps): half the variance's relative error
    ee = em + 2 * U * (e.abs() + s.abs())
    ev = sums * var + (2 * e.abs() * ee + ee * ee).mean(1, keepdim=True)
    rel = 0.5 * ev / (var + eps) + 6 * U
    en = q * ee + n.abs() * rel
    g = gamma.double() if gamma is not None else torch.ones(D, dtype=torch.float64, device=s.device)
    y = n * g + (beta.double() if beta is not None else 0)
    return s, y, en * g.abs() * (1 + 4 * U) + 3 * U * (n * g).abs() + 2 * U * y.abs()


def layernorm_bwd(s, dy, dsum, gamma, eps):
    """{name: (value, bound)}"""
    s, dy = s.double(), dy.double()
    D, M = s.shape[1], s.shape[0]
    sums = (D / 64 + 14) * U
    em = (sums + U) * s.abs().mean(1, keepdim=True)
    e = s - s.mean(1, keepdim=True)
    var = (e * e).mean(1, keepdim=True)
    q = 1 / torch.sqrt(var + eps)
    n = e * q
    ee = em + 2 * U * (e.abs() + s.abs())
    ev = sums * var + (2 * e.abs() * ee + ee * ee).mean(1, keepdim=True)
    rel = 0.5 * ev / (var + eps) + 6 * U
    en = q * ee + n.abs() * rel
    g = dy * gamma.double() if gamma is not None else dy
    level, along = g.mean(1, keepdim=True), (g * n).mean(1, keepdim=True)
    el = (sums + 2 * U) * g.abs().mean(1, keepdim=True)
    ea = (g.abs() * en).mean(1, keepdim=True) + (sums + 4 * U) * (g * n).abs().mean(1, keepdim=True) + rel * along.abs()
    dx = q * (g - level - n * along)
    mag = g.abs() + level.abs() + (n * along).abs()
    err = q * (el + n.abs() * ea + en * along.abs() + 6 * U * mag) + rel * q * mag
    if dsum is not None:
        dx = dx + dsum.double()
        err = err + 2 * U * dsum.double().abs()
    # a workgroup's rows (all of them where one wave takes them), then up to 1024 parts in 16 sums
    adds = (M / 4 + 100) * U
    return {"dx": (dx, err + 2 * U * dx.abs()),
            "dgamma": ((dy * n).sum(0), (dy.abs() * en).sum(0) + adds * (dy.abs() * (n.abs() + en)).sum(0)),
            "dbeta": (dy.sum(0), adds * dy.abs().sum(0))}


def act(z, name):
    """(act(z), act'(z), a bound on |act'|'s own error per unit of roundings); name as xema_act."""
    return (z, torch.ones_like(z)) if name == 2 else activation(z, name)


def linear(x, w, bias, name, resid):
    """(z, bound, y, bound of y before its rounding)"""
    z, ez = product(x, w, 2)
    if bias is not None:
        z, ez = z + bias.double(), ez + 2 * U * bias.double().abs()
    ez = ez + 2 * U * z.abs()
    a, _ = act(z, name)
    # |act'| is at most 1.13; the sigmoid's argument and value are off by a few units of |z| U
    ea = ez if name == 2 else 1.13 * ez + 16 * U * z.abs() * (1 + z.abs().clamp(max=100.0) * 0.3) + 4 * U * a.abs()
    y = a + resid.double() if resid is not None else a
    return z, ez, y, ea + 2 * U * y.abs()


def linear_bwd(x, w, z, dy, name, dtype):
    """{name: (value, bound before its rounding)} given the kept z"""
    x, w, dy = x.double(), w.double(), dy.double()
    M, N = dy.shape
    if name == 2:
        dz, ez = dy, torch.zeros_like(dy)
    else:
        dz = dy * act(z.double(), name)[1]
        ez = dy.abs() * 1.13 * 32 * U * (1 + z.double().abs().clamp(max=100.0))
    rz = rounded(dz, ez, dtype)       # (none where dy is dz and has the type already: then less than that)
    return {"dx": (dz @ w, rz @ w.abs() + (N + 24) * 2 * U * ((dz.abs() + rz) @ w.abs())),
            "dw": (dz.t().contiguous() @ x, rz.t() @ x.abs() + (M + 24) * 2 * U * ((dz.abs() + rz).t() @ x.abs())),
            "dbias": (dz.sum(0), ez.sum(0) + (M + 4) * U * (dz.abs() + ez).sum(0))}


# The exponential's results below fp32's normal range are zeros: a weight is off by up to its least normal value.
FLUSH = 2.0 ** -126


def _heads(t, batch, heads, d):
    """[batch * n, heads * d] to [batch, heads, n, d] in 64 bits"""
    return t.double().reshape(batch, -1, heads, d).transpose(1, 2).contiguous()


def _flat(t):
    b, h, n, d = t.shape
    return t.transpose(1, 2).reshape(b * n, h * d)


def _scores(q, k, lens, scale):
    """s (-inf where no state is), the bound on an exponent s_ij - m_i's error, and which are there"""
    S, d = k.shape[2], k.shape[3]
    kt = k.transpose(2, 3).contiguous()
    s, mag = q @ kt * scale, q.abs() @ kt.abs() * scale
    there = (torch.arange(S, device=q.device)[None] < lens[:, None])[:, None, None, :]
    # the products' sum (an MFMA truncates: 2 U an addition); scale * log2(e), its product and the difference
    e = (d + 2) * 2 * U * mag + 8 * U * s.abs()
    e = torch.where(there, e, 0.0)
    s = torch.where(there, s, -math.inf)
    return s, e.amax(3, keepdim=True) + 16 * U, there


def attention(q, k, v, batch, heads, kv_heads, d, lens, scale, dtype):
    """{name: (value, bound before its rounding)}: o [batch * q_len, heads * d] and lse [batch, heads, q_len]"""
    q = _heads(q, batch, heads, d)
    k, v = (_heads(t, batch, kv_heads, d).repeat_interleave(heads // kv_heads, 1) for t in (k, v))
    v = torch.where((torch.arange(k.shape[2], device=q.device)[None] < lens[:, None])[:, None, :, None], v, 0.0)
    k = torch.where((torch.arange(k.shape[2], device=q.device)[None] < lens[:, None])[:, None, :, None], k, 0.0)
    s, e, _ = _scores(q, k, lens, scale)
    S = k.shape[2]
    m = s.amax(3, keepdim=True).clamp(min=-1e300)
    w = torch.exp(s - m)
    total = w.sum(3, keepdim=True)
    p = w / total.clamp(min=1e-300)
    sums = (S + 100) * 2 * U         # in tiles, lanes and parts
    rel = 2 * e + sums               # numerator and denominator
    o = p @ v
    # each weight is rounded to the type, the largest being at least 1 beside what fp16 cannot hold
    ep = p * (rel + HALF[dtype]) * (1 + rel) + TINY[dtype] + FLUSH
    err = ep @ v.abs() + sums * ((p + ep) @ v.abs())
    lse = (m + torch.log(total))[..., 0]
    return {"o": (_flat(o), _flat(err) + 2 * U * _flat(o).abs()), "lse": (lse, (rel[..., 0] + 4 * U * lse.abs() + 16 * U))}


def attention_bwd(q, k, v, o, lse, do, batch, heads, kv_heads, d, lens, scale, dtype):
    """{dq, dk, dv: (value, bound before its rounding)}, given o and lse as stored"""
    group = heads // kv_heads
    q, o, do = (_heads(t, batch, heads, d) for t in (q, o, do))
    k, v = (_heads(t, batch, kv_heads, d) for t in (k, v))
    S, L = k.shape[2], q.shape[2]
    there = (torch.arange(S, device=q.device)[None] < lens[:, None])[:, None, :, None]
    k, v = (torch.where(there, t, 0.0).repeat_interleave(group, 1) for t in (k, v))
    s, e, _ = _scores(q, k, lens, scale)
    lse = lse.double()[..., None]
    p = torch.where(torch.isinf(s), 0.0, torch.exp(s - torch.where(torch.isinf(lse), 0.0, lse)))
    rp = e + 4 * U * torch.where(torch.isinf(lse), 0.0, lse).abs() + 32 * U
    D, mag_d = (do * o).sum(3, keepdim=True), (do * o).abs().sum(3, keepdim=True)
    vt = v.transpose(2, 3).contiguous()
    dp, mag = do @ vt, do.abs() @ vt.abs()
    ds = p * (dp - D)
    e_dp = (d + 4) * 2 * U * (mag + mag_d) + 4 * U * (dp.abs() + D.abs())
    e_ds = ds.abs() * rp + p * (1 + rp) * e_dp + FLUSH * (dp.abs() + D.abs() + e_dp)
    r_ds = torch.where(p > 0, rounded(ds, e_ds, dtype), 0.0)
    # fp16 carries 2^14 p
    r_p = torch.where(p > 0, p * (rp + HALF[dtype]) * (1 + rp) + TINY[dtype] * 2.0 ** -14 + FLUSH, 0.0)
    dq, eq = ds @ k * scale, (r_ds @ k.abs() + (S + 60) * 2 * U * ((ds.abs() + r_ds) @ k.abs())) * scale

    def shared(t):
        return t.reshape(batch, kv_heads, group, S, d).sum(2)

    add = (L * group + 100) * 2 * U
    dst, rst, pt, rpt = (t.transpose(2, 3).contiguous() for t in (ds, r_ds, p, r_p))
    dk = shared(dst @ q) * scale
    ek = shared(rst @ q.abs() + add * ((dst.abs() + rst) @ q.abs())) * scale
    dv = shared(pt @ do)
    ev = shared(rpt @ do.abs() + add * ((pt + rpt) @ do.abs()))
    return {n: (_flat(t), _flat(x) + 4 * U * _flat(t).abs()) for n, t, x in (("dq", dq, eq), ("dk", dk, ek), ("dv", dv, ev))}
