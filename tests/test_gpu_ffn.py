"""The feed-forward sub-block's operators against their definitions in 64 bits:
odd sizes, leading dimensions with memory between the rows that must stay as it
was, every type, rows with and without adapters, NaN and infinities."""
import pytest
import torch

import ffn_reference as R
import paper_2607_11136_amd as X

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
CODE = {torch.bfloat16: X.XEMA_BF16, torch.float16: X.XEMA_F16, torch.float32: X.XEMA_F32, torch.float8_e4m3fn: X.XEMA_E4M3}
BF16, F16, F32, E4M3 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def normal(g, shape, std=1.0, dtype=BF16, mean=0.0):
    return (torch.randn(shape, generator=g, device=DEV) * std + mean).to(dtype)


def strided(t, gap):
    """`t` in rows `gap` elements further apart, the gap holding a pattern; (matrix view, whole buffer)."""
    rows, width = t.shape
    buf = torch.full((rows, width + gap), 3.0, device=DEV).to(t.dtype)
    buf[:, :width] = t
    return buf[:, :width], buf


def empty(rows, width, gap, dtype):
    """An output to write: NaN bytes, the gap between its rows checked by `gap_kept`."""
    buf = torch.empty((rows, width + gap), dtype=dtype, device=DEV)
    buf.view(torch.uint8).fill_(0xFF)
    return buf


def gap_kept(buf, width):
    n = buf.element_size()
    assert bool((buf.view(torch.uint8).view(buf.shape[0], -1)[:, width * n:] == 0xFF).all())


def ld(t):
    return t.stride(0)


# -- RMS norm ----------------------------------------------------------------------------------------------------


def run_norm(x, resid, gamma, eps, y, dim, sum=None, y_scale=None, stream=None):
    X.xema_op_rmsnorm(X.rmsnorm_args(x, CODE[x.dtype], x.shape[0], dim, gamma, eps, y, CODE[y.dtype], y_scale=y_scale, resid=resid,
                                     resid_dtype=CODE[resid.dtype] if resid is not None else 0, sum=sum,
                                     sum_dtype=CODE[sum.dtype] if sum is not None else 0, ldx=ld(x),
                                     ld_resid=ld(resid) if resid is not None else 0, ld_sum=ld(sum) if sum is not None else 0,
                                     ldy=ld(y)), stream)


def check_e4m3(y, scale, want, rel, what):
    """Codes and scales of `want`, off by at most rel before their rounding."""
    top = want.abs().amax(1)
    lo, hi = (torch.exp2(torch.ceil(torch.log2((top * f).clamp(min=1e-300) / 448)).clamp(min=-126)) for f in (1 - 2 * rel, 1 + 2 * rel))
    s = scale.double()
    assert bool(((s == lo) | (s == hi)).all()), what
    v = want / s[:, None]
    R.within(y.float(), v, R.e4m3_steps(v.abs() * (1 + rel)) * (1 + 1e-12) + rel * v.abs(), what)


@pytest.mark.parametrize("rows,dim", [(1, 8), (1, 16384), (2, 16), (3, 256), (5, 504), (4, 512), (7, 520), (130, 1368), (9, 2048), (6, 2056),
                                      (33, 4096), (2, 8200)])
@pytest.mark.parametrize("xt,rt,yt", [(BF16, None, BF16), (F16, F32, F16), (F32, F32, BF16), (BF16, BF16, F16), (F32, None, F16),
                                      (F16, F16, BF16)])
def test_rmsnorm(rows, dim, xt, rt, yt):
    g = gen(rows * 7 + dim)
    x, _ = strided(normal(g, (rows, dim), 2.0, xt), 8)
    resid = strided(normal(g, (rows, dim), 3.0, rt), 16)[0] if rt else None
    gamma = normal(g, (dim,), 0.3, mean=1.0) if dim % 16 else None
    y, s = empty(rows, dim, 24, yt), empty(rows, dim, 8, rt or F32)
    run_norm(x, resid, gamma, 1e-5, y, dim, s)
    want_s, want, rel = R.rmsnorm(x, resid, gamma, 1e-5)
    R.within(y[:, :dim], want, R.rounded(want, rel * want.abs(), yt), "y")
    R.within(s[:, :dim], want_s, R.rounded(want_s, R.U * want_s.abs(), s.dtype), "sum")
    gap_kept(y, dim)
    gap_kept(s, dim)


@pytest.mark.parametrize("rows,dim", [(1, 16), (4, 4096), (3, 16384), (65, 1552), (257, 512)])
@pytest.mark.parametrize("xt", [BF16, F16, F32])
def test_rmsnorm_8bit(rows, dim, xt):
    g = gen(rows + dim)
    size = torch.exp(4 * torch.randn((rows, 1), generator=g, device=DEV)).clamp(1e-3, 1e3)
    x = (torch.randn((rows, dim), generator=g, device=DEV) * size).to(xt)
    resid = normal(g, (rows, dim), 1.0, F32)
    gamma = normal(g, (dim,), 0.3, mean=1.0)
    y, scale = empty(rows, dim, 16, E4M3), torch.full((rows,), -1.0, device=DEV)
    run_norm(x, resid, gamma, 1e-6, y, dim, None, scale)
    _, want, rel = R.rmsnorm(x, resid, gamma, 1e-6)
    check_e4m3(y[:, :dim], scale, want, rel, "codes")
    gap_kept(y, dim)


def test_rmsnorm_8bit_scale_is_the_smallest_power_of_two():
    """Rows whose largest value is exactly 448 * 2^k, or the next fp32 value
    above it: eps is far above the squares, so y = s / sqrt(eps) = s."""
    dim = 512
    rows = []
    for k in range(-20, -14):
        for top in (448.0 * 2.0 ** k, float(torch.nextafter(torch.tensor(448.0 * 2.0 ** k), torch.tensor(1e9)))):
            r = torch.zeros(dim)
            r[3], r[4] = -top, top * 2.0 ** -12
            rows.append(r)
    # y = s / sqrt(mean s^2 + eps): mean s^2 <= 2 * (448 * 2^-14)^2 / 512 = 3e-6 < 2^-25 * 2^7; eps = 2^40 leaves it out of the sum
    x = torch.stack(rows).to(DEV) * 2.0 ** 20
    y, scale = empty(len(rows), dim, 0, E4M3), torch.empty(len(rows), device=DEV)
    run_norm(x, None, None, 2.0 ** 60, y, dim, None, scale)
    s = x.double() * 2.0 ** -30
    want = torch.exp2(torch.ceil(torch.log2(s.abs().amax(1) / 448)))
    assert torch.equal(scale.double(), want)
    v = s / want[:, None]
    R.within(y.float(), v, R.e4m3_steps(v) * (1 + 1e-6), "codes")


@pytest.mark.parametrize("dim", [512, 4096])
def test_rmsnorm_zero_rows_and_non_finite_rows(dim):
    x = normal(gen(1), (6, dim), 1.0, F32)
    x[1] = 0
    x[2, 5] = float("inf")
    x[3, 7] = float("nan")
    x[4, dim - 1] = float("-inf")
    y, scale = empty(6, dim, 0, E4M3), torch.zeros(6, device=DEV)
    run_norm(x, None, None, 1e-6, y, dim, None, scale)
    assert torch.isnan(scale).tolist() == [False, False, True, True, True, False]
    assert bool((y[1].float() == 0).all()) and scale[1] == 2.0 ** -126
    assert bool(torch.isnan(y[2:5].float()).all())
    want = R.rmsnorm(x, None, None, 1e-6)
    for r in (0, 5):
        check_e4m3(y[r:r + 1], scale[r:r + 1], want[1][r:r + 1], want[2], "finite rows")
    # 16 bits: the formula's values, an infinity's own place NaN and zeros beside it
    y16 = empty(6, dim, 0, BF16)
    run_norm(x, None, None, 1e-6, y16, dim)
    assert torch.isnan(y16[2]).nonzero()[:, 0].tolist() == [5] and bool((y16[2][torch.arange(dim, device=DEV) != 5] == 0).all())
    assert bool(torch.isnan(y16[3]).all()) and not bool(torch.isnan(y16[[0, 1, 5]]).any())


def test_rmsnorm_updates_the_residual_in_place():
    g = gen(5)
    x, resid = normal(g, (37, 1536)), normal(g, (37, 1536), 2.0, F32)
    kept = resid.clone()
    y, s = empty(37, 1536, 0, BF16), empty(37, 1536, 0, F32)
    run_norm(x, kept, None, 1e-6, y, 1536, s)
    y2 = empty(37, 1536, 0, BF16)
    run_norm(x, resid, None, 1e-6, y2, 1536, resid)
    assert torch.equal(y, y2) and torch.equal(s, resid)


@pytest.mark.parametrize("rows,dim", [(1, 8), (1, 4096), (3, 512), (17, 520), (130, 2048), (6, 2056), (2500, 1032), (300, 8192), (5, 16384)])
@pytest.mark.parametrize("st,dt,ot", [(BF16, BF16, BF16), (F16, F16, F16), (F32, BF16, F32), (BF16, F32, F16), (F32, F16, BF16)])
def test_rmsnorm_bwd(rows, dim, st, dt, ot):
    g = gen(rows + 3 * dim)
    s, dy = strided(normal(g, (rows, dim), 2.0, st), 8)[0], strided(normal(g, (rows, dim), 0.5, dt), 16)[0]
    gamma = normal(g, (dim,), 0.3, mean=1.0)
    dsum = normal(g, (rows, dim), 0.5, ot) if rows % 2 else None
    dx, dgamma = empty(rows, dim, 8, ot), empty(1, dim, 0, F32)[0]
    n = X.xema_rmsnorm_bwd_workspace_bytes(rows, dim)
    ws = empty(1, n, 0, torch.uint8)[0]
    X.xema_op_rmsnorm_bwd(X.rmsnorm_bwd_args(s, CODE[st], rows, dim, gamma, 1e-5, dy, CODE[dt], dx, CODE[ot], dgamma, ws, n, dsum=dsum,
                                             dsum_dtype=CODE[ot], ld_s=ld(s), ld_dy=ld(dy), ld_dx=ld(dx)))
    want = R.rmsnorm_bwd(s, dy, dsum, gamma, 1e-5)
    v, e = want["dx"]
    R.within(dx[:, :dim], v, R.rounded(v, e, ot), "dx")
    R.within(dgamma, *want["dgamma"], "dgamma")
    gap_kept(dx, dim)


def test_rmsnorm_bwd_is_the_slope_of_the_forward():
    """Differences of the 64-bit forward along random directions."""
    g = gen(11)
    s, dy, gamma = normal(g, (5, 64), 1.0, F32), normal(g, (5, 64), 1.0, F32), normal(g, (64,), 0.3, mean=1.0)
    dx, dgamma = empty(5, 64, 0, F32), empty(1, 64, 0, F32)[0]
    n = X.xema_rmsnorm_bwd_workspace_bytes(5, 64)
    X.xema_op_rmsnorm_bwd(X.rmsnorm_bwd_args(s, X.XEMA_F32, 5, 64, gamma, 1e-5, dy, X.XEMA_F32, dx, X.XEMA_F32, dgamma,
                                             torch.empty(n, dtype=torch.uint8, device=DEV), n))
    loss = lambda s_, g_: (R.rmsnorm(s_, None, g_, 1e-5)[1] * dy.double()).sum()  # noqa: E731
    h = 1e-6
    for seed in range(4):
        v = torch.randn(s.shape, generator=gen(seed), device=DEV, dtype=torch.float64)
        slope = (loss(s.double() + h * v, gamma) - loss(s.double() - h * v, gamma)) / (2 * h)
        assert abs(float(slope - (dx.double() * v).sum())) < 1e-4 * (1 + float((dx.double() * v).abs().sum()))
        v = torch.randn(64, generator=gen(seed), device=DEV, dtype=torch.float64)
        slope = (loss(s, gamma.double() + h * v) - loss(s, gamma.double() - h * v)) / (2 * h)
        assert abs(float(slope - (dgamma.double() * v).sum())) < 1e-4 * (1 + float((dgamma.double() * v).abs().sum()))


@pytest.mark.parametrize("which", ["dy", "dsum", "s"])
def test_rmsnorm_bwd_in_place(which):
    g = gen(3)
    t = {n: normal(g, (50, 1024), 1.0, BF16) for n in ("s", "dy", "dsum")}
    out = {}
    for dx in (torch.empty_like(t["s"]), None):
        src = {n: v.clone() for n, v in t.items()}
        dx = src[which] if dx is None else dx
        X.xema_op_rmsnorm_bwd(X.rmsnorm_bwd_args(src["s"], 0, 50, 1024, None, 1e-6, src["dy"], 0, dx, 0, dsum=src["dsum"]))
        out[len(out)] = dx
    assert torch.equal(out[0], out[1])


# -- gated feed-forward ------------------------------------------------------------------------------------------

SIZES = [(1, 8, 8), (1, 4096, 1024), (2, 64, 40), (16, 72, 136), (17, 512, 1368), (32, 1096, 72), (33, 1096, 72), (63, 128, 64), (65, 136, 200), (130, 328, 520), (257, 1544, 264),
         (700, 256, 2056), (1500, 192, 4104), (582, 72, 3376), (2435, 88, 1552), (207, 64, 4208)]


def gated_inputs(rows, dim, hidden, dtype, bias, seed):
    g = gen(seed)
    x, _ = strided(normal(g, (rows, dim), 1.0, dtype), 8)
    wg, wu = normal(g, (hidden, dim), 2 * dim ** -0.5, dtype), normal(g, (hidden, dim), dim ** -0.5, dtype)
    bg, bu = (normal(g, (hidden,), 0.5), normal(g, (hidden,), 0.5)) if bias else (None, None)
    return x, wg, wu, bg, bu


def pack24(t):
    """[rows, 2 hidden] (g, then u) in fp32, rounded to 24 bits, as xema_op_gated_ffn stores them."""
    rows, hidden = t.shape[0], t.shape[1] // 2
    b = t.float().view(torch.int32)
    b = (b + 0x7F + ((b >> 8) & 1)) & -256
    q = b.view(rows, 2, hidden // 4, 4).transpose(1, 2).contiguous()      # [rows, groups, (g, u), 4]
    upper = ((q >> 16) & 0xFFFF).to(torch.int16).view(torch.uint8).view(rows, hidden // 4, 16)
    low = ((q >> 8) & 0xFF).to(torch.uint8).view(rows, hidden // 4, 8)
    return torch.cat((upper, low), 2).contiguous().view(rows, 6 * hidden)


def unpack24(pre, hidden):
    """What such bytes stand for, [rows, 2 hidden]."""
    p = pre.view(-1, hidden // 4, 24)
    rows = p.shape[0]
    upper = p[:, :, :16].contiguous().view(torch.int16).view(rows, -1, 2, 4).to(torch.int32)
    b = (upper << 16) | (p[:, :, 16:].contiguous().view(rows, -1, 2, 4).to(torch.int32) << 8)
    return b.view(torch.float32).transpose(1, 2).reshape(rows, 2 * hidden)


def empty_pre(rows, hidden):
    assert X.xema_gated_ffn_pre_bytes(rows, hidden) == 6 * rows * hidden
    return empty(rows, 6 * hidden, 0, torch.uint8)


def run_gated(x, wg, wu, bg, bu, act, y, pre=None, stream=None):
    rows, dim, hidden = x.shape[0], x.shape[1], wg.shape[0]
    X.xema_op_gated_ffn(X.gated_ffn_args(CODE[x.dtype], act, x, rows, dim, wg, wu, hidden, y, CODE[y.dtype], gate_b=bg, up_b=bu, pre=pre,
                                         ldx=ld(x), ldy=ld(y)), stream)


@pytest.mark.parametrize("rows,dim,hidden", SIZES)
@pytest.mark.parametrize("dtype,act,bias", [(BF16, 0, False), (F16, 1, True), (BF16, 1, True), (F16, 0, False)])
def test_gated_ffn(rows, dim, hidden, dtype, act, bias):
    x, wg, wu, bg, bu = gated_inputs(rows, dim, hidden, dtype, bias, rows + dim)
    y, pre = empty(rows, hidden, 16, dtype), empty_pre(rows, hidden)
    run_gated(x, wg, wu, bg, bu, act, y, pre)
    want, e, g, eg, u, eu = R.gated(x, wg, wu, bg, bu, act)
    R.within(y[:, :hidden], want, R.rounded(want, e, dtype), "y")
    kept = unpack24(pre, hidden)
    R.within(kept[:, :hidden], g, eg + 2.0 ** -16 * (g.abs() + eg), "g")
    R.within(kept[:, hidden:], u, eu + 2.0 ** -16 * (u.abs() + eu), "u")
    gap_kept(y, hidden)
    y2 = empty(rows, hidden, 0, dtype)
    run_gated(x, wg, wu, bg, bu, act, y2)
    assert torch.equal(y2, y[:, :hidden])


SIZES_8BIT = [(1, 16, 8), (1, 4096, 1024), (3, 144, 40), (16, 2064, 24), (31, 1040, 72), (65, 272, 200), (130, 336, 520), (700, 128, 2056),
              (1500, 512, 4104), (582, 80, 3376), (2435, 144, 1552), (207, 64, 4208)]

# A 16x16x128 MFMA of e4m3 values aligns its 128 products to the largest before
# it adds them: off by up to 2^-14 of the sum of their magnitudes (measured 2^-14.8).
E4M3_SUM = 2.0 ** -14


@pytest.mark.parametrize("rows,dim,hidden", SIZES_8BIT)
@pytest.mark.parametrize("yt,act,bias", [(BF16, 0, False), (F16, 1, True)])
def test_gated_ffn_8bit(rows, dim, hidden, yt, act, bias):
    x, wg, wu, bg, bu = gated_inputs(rows, dim, hidden, F32, bias, rows + dim)
    q, scale = [], []
    for t in (x, wg, wu):
        s = t.abs().amax(1) / 448
        q.append((t / s[:, None]).to(E4M3))
        scale.append(s)
    xq, _ = strided(q[0].float(), 16)
    xq = xq.to(E4M3)
    y = empty(rows, hidden, 8, yt)
    X.xema_op_gated_ffn(X.gated_ffn_args(X.XEMA_E4M3, act, xq, rows, dim, q[1], q[2], hidden, y, CODE[yt], gate_b=bg, up_b=bu,
                                         x_scale=scale[0], gate_scale=scale[1], up_scale=scale[2], ldx=ld(xq), ldy=ld(y)))
    v = [a.double() * s.double()[:, None] for a, s in zip(q, scale)]
    want, e, *_ = R.gated(v[0], v[1], v[2], bg, bu, act, slack=E4M3_SUM)
    R.within(y[:, :hidden], want, R.rounded(want, e, yt), "y")
    gap_kept(y, hidden)


@pytest.mark.parametrize("act", [0, 1])
def test_gated_ffn_extreme_gates(act):
    """Gates from -1e30 to 1e30 reach the activation's limits without a NaN."""
    gates = [-1e30, -1e5, -200.0, -90.0, -30.0, -1.0, 0.0, 1.0, 30.0, 90.0, 200.0, 1e5, 1e30]
    x = torch.zeros((1, 16), device=DEV, dtype=BF16)
    x[0, :2] = 1
    wg, wu = torch.zeros((16, 16), device=DEV, dtype=BF16), torch.zeros((16, 16), device=DEV, dtype=BF16)
    wg[:len(gates), 0] = torch.tensor(gates)
    wu[:, 1] = 1
    y, pre = empty(1, 16, 0, BF16), empty_pre(1, 16)
    run_gated(x, wg, wu, None, None, act, y, pre)
    g = wg[:, 0].double()
    a, slope = R.activation(g, act)
    R.within(y[0], a, R.rounded(a, 64 * R.U * a.abs() + 1e-30, BF16), "act")
    dy = torch.ones((1, 16), device=DEV, dtype=BF16)
    n = X.xema_gated_ffn_bwd_workspace_bytes(1, 16, 16)
    dgb, dub = torch.empty(16, device=DEV, dtype=BF16), torch.empty(16, device=DEV, dtype=BF16)
    X.xema_op_gated_ffn_bwd(X.gated_ffn_bwd_args(X.XEMA_BF16, act, x, 1, 16, wg, wu, 16, pre, dy, None, None, None,
                                                 torch.empty(n, dtype=torch.uint8, device=DEV), n, dgate_b=dgb, dup_b=dub))
    slope = torch.where(g.abs() > 1e4, (g > 0).double(), slope)     # (the definition's own terms overflow there)
    R.within(dgb, slope, R.rounded(slope, 1e-5 * slope.abs() + 1e-8, BF16), "slope")
    R.within(dub, a, R.rounded(a, 64 * R.U * a.abs() + 1e-30, BF16), "act again")


BWD_SIZES = [(4500, 64, 72), (9000, 72, 328), (2100, 264, 392), (1, 8, 8), (2, 64, 40), (17, 512, 1368), (63, 128, 64), (65, 136, 200), (130, 328, 520), (257, 1544, 264), (1100, 256, 1032),
             (2100, 4104, 2056), (5000, 4104, 72), (70, 136, 4104), (5, 1032, 2056),
             (39, 280, 5456), (35, 544, 5504), (33, 528, 1816), (2711, 1456, 72), (1614, 1240, 2400),
             (40, 1800, 2304), (69, 1136, 4120)]


def run_bwd(x, wg, wu, pre, dy, act, bias=True, dx=True, dw=True, gap=8, stream=None):
    rows, dim, hidden = x.shape[0], x.shape[1], wg.shape[0]
    t = x.dtype
    out = {"dx": empty(rows, dim, gap, t) if dx else None, "dgate_w": empty(hidden, dim, 0, t) if dw else None,
           "dup_w": empty(hidden, dim, 0, t) if dw else None, "dgate_b": empty(1, hidden, 0, BF16)[0] if bias else None,
           "dup_b": empty(1, hidden, 0, BF16)[0] if bias else None}
    n = X.xema_gated_ffn_bwd_workspace_bytes(rows, dim, hidden)
    ws = empty(1, n, 0, torch.uint8)[0]
    X.xema_op_gated_ffn_bwd(X.gated_ffn_bwd_args(CODE[t], act, x, rows, dim, wg, wu, hidden, pre, dy, out["dx"], out["dgate_w"], out["dup_w"],
                                                 ws, n, dgate_b=out["dgate_b"], dup_b=out["dup_b"], ldx=ld(x), ld_dy=ld(dy),
                                                 ld_dx=ld(out["dx"]) if dx else 0), stream)
    out["ws"] = ws
    return out


@pytest.mark.parametrize("rows,dim,hidden", BWD_SIZES)
@pytest.mark.parametrize("dtype,act", [(BF16, 0), (F16, 1)])
def test_gated_ffn_bwd(rows, dim, hidden, dtype, act):
    x, wg, wu, _, _ = gated_inputs(rows, dim, hidden, dtype, False, rows + dim)
    g = gen(rows)
    kept = unpack24(pack24(normal(g, (rows, 2 * hidden), 1.5, F32)), hidden)
    pre, dy = pack24(kept), strided(normal(g, (rows, hidden), 0.5, dtype), 24)[0]
    out = run_bwd(x, wg, wu, pre, dy, act)
    want = R.gated_bwd(x, wg, wu, kept, dy, act, dtype)
    for n in ("dgate_b", "dup_b", "dx", "dgate_w", "dup_w"):
        v, e = want[n]
        got = out[n][:, :dim] if n == "dx" else out[n]
        R.within(got, v, R.rounded(v, e, got.dtype), n)
    gap_kept(out["dx"], dim)
    for kw in ({"bias": False, "dx": False}, {"bias": False, "dw": False}, {"dx": False, "dw": False}):
        part = run_bwd(x, wg, wu, pre, dy, act, **kw)
        for n, v in part.items():
            if v is not None and n not in ("ws", "dx"):
                assert torch.equal(v, out[n]), (n, kw)
            if v is not None and n == "dx":
                assert torch.equal(v[:, :dim], out["dx"][:, :dim])


def test_gated_ffn_bwd_is_the_slope_of_the_forward():
    """Differences of the 64-bit forward, along random directions of every input."""
    rows, dim, hidden, act = 12, 64, 40, 0
    x, wg, wu, bg, bu = gated_inputs(rows, dim, hidden, F16, True, 1)
    x = x.contiguous()
    dy = normal(gen(2), (rows, hidden), 1.0, F16)
    y, pre = empty(rows, hidden, 0, F16), empty_pre(rows, hidden)
    run_gated(x, wg, wu, bg, bu, act, y, pre)
    out = run_bwd(x, wg, wu, pre, dy, act, gap=0)
    names = {"dx": 0, "dgate_w": 1, "dup_w": 2, "dgate_b": 3, "dup_b": 4}
    at = [t.double() for t in (x, wg, wu, bg, bu)]
    loss = lambda a: (R.gated(*a, act)[0] * dy.double()).sum()  # noqa: E731
    h = 1e-6
    for n, i in names.items():
        v = torch.randn(at[i].shape, generator=gen(i), device=DEV, dtype=torch.float64)
        up, down = list(at), list(at)
        up[i], down[i] = at[i] + h * v, at[i] - h * v
        slope = float((loss(up) - loss(down)) / (2 * h))
        # roundings: dg and du, and the result, half a step each in the sum of magnitudes (and pre's, far below)
        most = float((out[n].double() * v).abs().sum())
        half = R.HALF[out[n].dtype if n.endswith("_b") else F16]
        assert abs(slope - float((out[n].double() * v).sum())) < 4 * half * most + 1e-5, n


def test_gated_ffn_bwd_no_rows():
    x, wg, wu, _, _ = gated_inputs(1, 64, 40, BF16, False, 1)
    z = torch.empty((0, 80), device=DEV, dtype=BF16)
    out = {n: empty(40, 64, 0, BF16) for n in ("dgate_w", "dup_w")}
    b = [empty(1, 40, 0, BF16)[0] for _ in range(2)]
    n = X.xema_gated_ffn_bwd_workspace_bytes(0, 64, 40)
    X.xema_op_gated_ffn_bwd(X.gated_ffn_bwd_args(0, 0, x, 0, 64, wg, wu, 40, x, x, None, out["dgate_w"], out["dup_w"],
                                                 torch.empty(n, dtype=torch.uint8, device=DEV), n, dgate_b=b[0], dup_b=b[1]))
    for t in (*out.values(), *b):
        assert bool((t == 0).all())
    assert z.numel() == 0
    dgamma = empty(1, 64, 0, F32)[0]
    n = X.xema_rmsnorm_bwd_workspace_bytes(0, 64)
    X.xema_op_rmsnorm_bwd(X.rmsnorm_bwd_args(x, 0, 0, 64, None, 1e-6, x, 0, x, 0, dgamma, torch.empty(n, dtype=torch.uint8, device=DEV), n))
    assert bool((dgamma == 0).all())


# -- the shared projection with adapters -------------------------------------------------------------------------


def lora_inputs(rows, dim, out_dim, rank, n, dtype, seed, bias=True):
    g = gen(seed)
    return {"x": strided(normal(g, (rows, dim), 1.0, dtype), 8)[0], "w": normal(g, (out_dim, dim), dim ** -0.5, dtype),
            "bias": normal(g, (out_dim,), 0.5) if bias else None, "a": normal(g, (n, rank, dim), dim ** -0.5, dtype),
            "b": normal(g, (n, out_dim, rank), rank ** -0.5, dtype), "scale": torch.rand(n, generator=g, device=DEV) + 0.5}


def run_lora(d, ids, y, stream=None, n=None):
    rows, dim, out_dim, rank = d["x"].shape[0], d["x"].shape[1], d["w"].shape[0], d["a"].shape[1]
    n = d["a"].shape[0] if n is None else n
    nb = X.xema_lora_workspace_bytes(rows, rank)
    ws = empty(1, nb, 0, torch.uint8)[0]
    X.xema_op_lora_linear(X.lora_args(CODE[d["x"].dtype], d["x"], rows, dim, d["w"], out_dim, d["bias"], d["a"] if n else None,
                                      d["b"] if n else None, d["scale"] if n else None, rank, n, ids, y, CODE[y.dtype], ws, nb,
                                      ldx=ld(d["x"]), ldy=ld(y)), stream)
    return ws


def spread_ids(rows, n, how, seed):
    g = gen(seed)
    if how == "one":
        return torch.full((rows,), n - 1, dtype=torch.int32, device=DEV)
    if how == "runs":     # requests of unlike lengths, some without an adapter, padding behind
        cuts = torch.sort(torch.randint(0, rows + 1, (5,), generator=g, device=DEV)).values.tolist()
        ids = torch.full((rows,), -2, dtype=torch.int32, device=DEV)
        for i, (lo, hi) in enumerate(zip([0] + cuts, cuts)):
            ids[lo:hi] = i % (n + 1) - 1
        return ids
    return torch.randint(-2, n, (rows,), generator=g, device=DEV, dtype=torch.int32)     # every row its own


LORA_SIZES = [(1, 8, 8, 8, 1), (1, 4096, 1032, 16, 3), (5, 72, 136, 8, 2), (48, 512, 1024, 16, 20), (65, 136, 200, 24, 4), (130, 328, 520, 64, 7),
              (257, 1544, 264, 128, 5), (700, 256, 2056, 32, 40), (1500, 192, 4104, 8, 3), (9000, 256, 1544, 16, 4),
              (12500, 136, 520, 32, 5), (16, 2056, 72, 32, 3), (33, 1032, 88, 128, 2),
              (7, 264, 4360, 16, 3), (20, 136, 4136, 24, 4), (47, 72, 8192, 8, 2), (64, 520, 4104, 40, 9), (64, 2056, 520, 16, 3), (30, 64, 8200, 8, 2),
              (582, 72, 3376, 8, 2), (2100, 72, 136, 16, 6), (1100, 72, 136, 32, 6), (600, 136, 72, 64, 9), (4200, 136, 72, 64, 9),
              (4200, 264, 72, 128, 3), (1, 136, 8200, 16, 2), (13, 1032, 8264, 64, 5), (16, 64, 16392, 8, 30), (32, 520, 8328, 128, 6),
              (12400, 72, 72, 72, 4)]


@pytest.mark.parametrize("rows,dim,out_dim,rank,n", LORA_SIZES)
@pytest.mark.parametrize("how", ["one", "runs", "mixed"])
@pytest.mark.parametrize("dtype,yt", [(BF16, BF16), (F16, F16), (BF16, F16)])
def test_lora_linear(rows, dim, out_dim, rank, n, how, dtype, yt):
    d = lora_inputs(rows, dim, out_dim, rank, n, dtype, rows + dim, bias=rows % 2 == 1)
    ids = spread_ids(rows, n, how, rows)
    y = empty(rows, out_dim, 16, yt)
    before = y.clone()
    run_lora(d, ids, y)
    want, e = R.lora(d["x"], d["w"], d["bias"], d["a"], d["b"], d["scale"], ids, dtype)
    live = ids >= -1
    R.within(y[live][:, :out_dim], want[live], R.rounded(want, e, yt)[live], "y")
    assert torch.equal(y[~live].view(torch.int16), before[~live].view(torch.int16))
    gap_kept(y, out_dim)


def test_lora_adapters_do_not_touch_each_other():
    """One adapter of infinities and NaN: only the rows that name it see them;
    an id past the last one gives a row of NaN and touches no other."""
    for rows, how in ((40, "mixed"), (300, "mixed"), (600, "runs")):
        d = lora_inputs(rows, 264, 392, 16, 3, BF16, rows)
        ids = spread_ids(rows, 3, how, rows)
        ids[rows // 2] = 3
        ids[rows // 3] = 1 << 30
        good = empty(rows, 392, 0, BF16)
        run_lora(d, ids, good)
        assert bool(torch.isnan(good[ids >= 3]).all())
        d["a"][1, :, 5] = float("inf")
        d["b"][1, 7, :] = float("nan")
        d["b"][1, 9, 2] = float("-inf")
        got = empty(rows, 392, 0, BF16)
        run_lora(d, ids, got)
        other = (ids != 1) & (ids >= -1) & (ids < 3)
        assert torch.equal(got[other], good[other]) and bool(torch.isfinite(got[other]).all())
        if bool((ids == 1).any()):
            assert bool(torch.isnan(got[ids == 1][:, 7]).all())


@pytest.mark.parametrize("rows,rank", [(1, 8), (40, 16), (300, 64), (5000, 8)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_lora_infinities_follow_the_formula(rows, rank, dtype):
    """All weights positive: a row with an infinity is infinity in every column,
    not NaN, and so is one whose x a^T leaves the type's range."""
    d = lora_inputs(rows, 264, 392, rank, 2, dtype, rows)
    for n in ("x", "w", "a", "b"):
        d[n] = d[n].abs() + 2.0 ** -10
    ids = spread_ids(rows, 2, "mixed", rows)
    ids[0], ids[2:3] = 1, 0                    # (in both calls: a padding row would stay NaN)
    good, got = empty(rows, 392, 0, dtype), empty(rows, 392, 0, dtype)
    run_lora(d, ids, good)
    d["x"][0, 5] = float("inf")
    if rows > 2:
        d["x"][2] = torch.finfo(dtype).max     # (264 of them against a's sum of 8 at least)
    run_lora(d, ids, got)
    for r in (0, 2)[:1 + (rows > 2)]:
        assert bool((got[r] == float("inf")).all())
        got[r] = good[r]
    live = ids >= -1
    assert torch.equal(got[live], good[live])


def test_lora_without_adapters_is_the_projection():
    d = lora_inputs(70, 264, 392, 8, 1, F16, 4)
    y = empty(70, 392, 0, F16)
    run_lora(d, torch.full((70,), -1, dtype=torch.int32, device=DEV), y, n=0)
    want, e = R.lora(d["x"], d["w"], d["bias"], d["a"][:0], d["b"][:0], d["scale"][:0], torch.full((70,), -1, device=DEV), F16)
    want[:] = d["x"].double() @ d["w"].double().t() + d["bias"].double()
    R.within(y, want, R.rounded(want, e, F16), "y")


def test_lora_all_rows_padding():
    d = lora_inputs(300, 64, 72, 8, 2, BF16, 4)
    y = empty(300, 72, 0, BF16)
    run_lora(d, torch.full((300,), -5, dtype=torch.int32, device=DEV), y)
    gap_kept(y, 0)
