"""The linear layer with bias, activation and residual, and its gradient, against
their definitions in 64 bits: widths that no tile divides, few rows, every tile,
types, leading dimensions, the residual updated in place."""
import pytest
import torch

import cross_reference as R
import paper_2607_11136_amd as X
from test_gpu_ffn import BF16, CODE, DEV, F16, F32, empty, gap_kept, gen, ld, normal, strided

pytestmark = pytest.mark.gpu

# rows, dim, out_dim: every few-row kernel and every tile (tests/test_cross_rules.py)
SIZES = [(1, 8, 8), (1, 4096, 136), (17, 264, 72), (33, 520, 4096), (64, 72, 1000), (5, 136, 4104), (20, 264, 8192), (40, 72, 6000), (50, 136, 4608),
         (3, 264, 8200), (30, 72, 12008), (65, 40, 8), (100, 264, 392), (700, 136, 520), (300, 136, 8200), (1100, 72, 3000), (2600, 520, 2056),
         (6000, 64, 4104), (130, 2056, 72), (9000, 264, 8200), (9000, 520, 2056), (2600, 520, 8200)]
# whole and split k of either product, one launch and two
BWD_SIZES = [(1, 8, 8), (7, 72, 136), (65, 136, 200), (333, 512, 1368), (70, 136, 8200), (4500, 64, 72), (1614, 1240, 2400), (3000, 1032, 4104),
             (257, 8200, 136), (16, 2056, 2056), (2100, 264, 264), (9000, 136, 1032), (1000, 136, 264), (2048, 136, 264), (8200, 520, 264),
             (1000, 2056, 264), (8200, 136, 2056), (1000, 4104, 264), (2048, 4104, 264), (8200, 2056, 264), (8200, 136, 8200), (8200, 264, 4104)]


def run(x, w, bias, act, y, resid=None, pre=None, stream=None):
    N, dim = w.shape
    X.xema_op_linear(X.linear_args(CODE[x.dtype], x, x.shape[0], dim, w, N, bias, act, y, CODE[y.dtype], resid=resid,
                                   resid_dtype=CODE[resid.dtype] if resid is not None else 0, pre=pre, ldx=ld(x),
                                   ld_resid=ld(resid) if resid is not None else 0, ldy=ld(y)), stream)


def run_bwd(x, w, pre, dy, act, dx, dw, db, stream=None, ws=None):
    N, dim = w.shape
    n = X.xema_linear_bwd_workspace_bytes(x.shape[0], dim, N)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV) if ws is None else ws
    X.xema_op_linear_bwd(X.linear_bwd_args(CODE[x.dtype], act, x, x.shape[0], dim, w, N, pre, dy, CODE[dy.dtype], dx, dw, db, ws, ws.numel(),
                                           ldx=ld(x), ld_dy=ld(dy), ld_dx=ld(dx) if dx is not None else 0), stream)


def unpack(pre, rows, width):
    """z from its 24 bits: per four columns four upper halves, then four third bytes."""
    b = pre.view(rows, width // 4, 12).to(torch.int32)
    hi = b[:, :, 0:8:2] | b[:, :, 1:8:2] << 8
    return ((hi << 16) | (b[:, :, 8:] << 8)).view(torch.float32).reshape(rows, width)


@pytest.mark.parametrize("rows,dim,out", SIZES)
@pytest.mark.parametrize("t,act,yt,rt", [(BF16, 2, F32, F32), (F16, 1, F16, None), (BF16, 0, BF16, BF16), (F16, 2, BF16, F16), (BF16, 1, F32, None)])
def test_linear(rows, dim, out, t, act, yt, rt):
    g = gen(rows + dim + out)
    x, _ = strided(normal(g, (rows, dim), 1.0, t), 8)
    w = normal(g, (out, dim), 1.5 * dim ** -0.5, t)
    bias = normal(g, (out,), 0.5) if act else None
    resid = strided(normal(g, (rows, out), 2.0, rt), 16)[0] if rt else None
    y = empty(rows, out, 24, yt)
    pre = torch.full((X.xema_linear_pre_bytes(rows, out),), 0xFF, dtype=torch.uint8, device=DEV) if act == 1 else None
    run(x, w, bias, act, y, resid, pre)
    z, ez, want, err = R.linear(x, w, bias, act, resid)
    R.within(y[:, :out], want, R.rounded(want, err, yt), "y")
    gap_kept(y, out)
    if pre is not None:      # 16 significant bits
        R.within(unpack(pre, rows, out), z, ez + 2.0 ** -16 * (z.abs() + ez) + 2.0 ** -134, "z")


@pytest.mark.parametrize("rows,dim,out", BWD_SIZES)
@pytest.mark.parametrize("t,act,dt", [(BF16, 1, BF16), (F16, 0, F16), (BF16, 2, BF16), (F16, 2, F32)])
def test_gradient(rows, dim, out, t, act, dt):
    g = gen(rows + dim + out)
    x, _ = strided(normal(g, (rows, dim), 1.0, t), 8)
    w = normal(g, (out, dim), 1.5 * dim ** -0.5, t)
    dy, _ = strided(normal(g, (rows, out), 0.5, dt), 16)
    z = pre = None
    if act != 2:
        pre = torch.empty(X.xema_linear_pre_bytes(rows, out), dtype=torch.uint8, device=DEV)
        run(x, w, None, act, empty(rows, out, 0, t), None, pre)
        z = unpack(pre, rows, out)
    dx, dw, db = empty(rows, dim, 24, t), empty(out, dim, 0, t), empty(1, out, 0, BF16)[0]
    run_bwd(x, w, pre, dy, act, dx, dw, db)
    want = R.linear_bwd(x, w, z, dy, act, t)
    R.within(dx[:, :dim], want["dx"][0], R.rounded(*want["dx"], t), "dx")
    R.within(dw, want["dw"][0], R.rounded(*want["dw"], t), "dw")
    R.within(db, want["dbias"][0], R.rounded(*want["dbias"], BF16), "dbias")
    gap_kept(dx, dim)
    # each gradient alone has the same bytes
    kept = [t_.clone() for t_ in (dx, dw, db)]
    for a, b, c in ((dx, None, None), (None, dw, None), (None, None, db), (dx, None, db)):
        for t_ in (dx, dw, db):
            t_.view(torch.uint8).fill_(0xFF)
        run_bwd(x, w, pre, dy, act, a, b, c)
        for t_, k, there in zip((dx, dw, db), kept, (a, b, c)):
            assert torch.equal(t_.view(torch.uint8), k.view(torch.uint8)) if there is not None else bool((t_.view(torch.uint8) == 0xFF).all())


@pytest.mark.parametrize("act", [0, 1])
def test_gradient_against_differences(act):
    """The formula's own gradient in 64 bits meets central differences of sum(dy * y)."""
    g = gen(3)
    x, w, b, dy = (torch.randn(n, generator=g, device=DEV, dtype=torch.float64) for n in ((3, 8), (16, 8), (16,), (3, 16)))
    z = x @ w.t() + b
    want = R.linear_bwd(x, w, z, dy, act, F32)

    def loss():
        return float((dy * R.act(x @ w.t() + b, act)[0]).sum())

    for t, name, at in ((x, "dx", (1, 3)), (w, "dw", (15, 7)), (w, "dw", (0, 2)), (b, "dbias", (4,))):
        v, ends = float(t[at]), []
        for h in (1e-4, -1e-4):
            t[at] = v + h
            ends.append(loss())
        t[at] = v
        assert abs((ends[0] - ends[1]) / 2e-4 - float(want[name][0][at])) < 1e-5


@pytest.mark.parametrize("rows", [3, 300])
@pytest.mark.parametrize("rt", [F32, BF16, F16])
def test_residual_updated_in_place(rows, rt):
    g = gen(rows)
    x, w, resid = normal(g, (rows, 264)), normal(g, (520, 264), 0.1), normal(g, (rows, 520), 1.0, rt)
    y = empty(rows, 520, 0, rt)
    run(x, w, None, 2, y, resid)
    run(x, w, None, 2, resid, resid)
    assert torch.equal(y, resid)


def test_non_finite_values_and_saturated_activations():
    x, w = torch.zeros((70, 64), device=DEV, dtype=BF16), torch.zeros((72, 64), device=DEV, dtype=BF16)
    x[:, 0] = 1
    w[:, 0] = torch.linspace(-3e4, 3e4, 72, device=DEV).to(BF16)
    w[3, 0], w[5, 0], w[6, 0] = float("inf"), float("-inf"), float("nan")
    dy = torch.ones((70, 72), device=DEV, dtype=BF16)
    for act in (0, 1):
        y, pre = empty(70, 72, 0, F32), torch.empty(3 * 70 * 72, dtype=torch.uint8, device=DEV)
        run(x, w, None, act, y, None, pre)
        z = w[:, 0].double()
        live = [i for i in range(72) if i not in (3, 5, 6)]
        R.within(y[9, live], torch.where(z > 0, z, 0.0)[live], 4 * R.U * z.abs()[live] + 1e-30, "y")
        assert float(y[9, 3]) == float("inf") and bool(torch.isnan(y[9, 6]))
        db = empty(1, 72, 0, BF16)[0]
        run_bwd(x, w, pre, dy, act, None, None, db)
        R.within(db[live], torch.where(z > 0, 70.0, 0.0).double()[live], torch.full((len(live),), 0.3, device=DEV, dtype=torch.float64), "dbias")


def test_no_rows():
    x, w, dy = torch.zeros((8, 64), device=DEV, dtype=BF16), torch.ones((72, 64), device=DEV, dtype=BF16), torch.ones((8, 72), device=DEV, dtype=BF16)
    dw, db = empty(72, 64, 0, BF16), empty(1, 72, 0, BF16)[0]
    n = X.xema_linear_bwd_workspace_bytes(0, 64, 72)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    y = empty(8, 72, 0, BF16)
    X.xema_op_linear(X.linear_args(0, x, 0, 64, w, 72, None, 2, y, 0))
    X.xema_op_linear_bwd(X.linear_bwd_args(0, 2, x, 0, 64, w, 72, None, dy, 0, None, dw, db, ws, n))
    assert bool((dw == 0).all()) and bool((db == 0).all())
    gap_kept(y, 0)
