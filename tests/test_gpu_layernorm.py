"""Layer norm with the residual's addition and its gradient against their
definitions in 64 bits: odd sizes, every type, leading dimensions with memory
between the rows that must stay as it was, outputs that are an input."""
import pytest
import torch

import cross_reference as R
import paper_2607_11136_amd as X
from test_gpu_ffn import BF16, CODE, DEV, F16, F32, empty, gap_kept, gen, ld, normal, strided

pytestmark = pytest.mark.gpu

SIZES = [(1, 8), (1, 16384), (2, 16), (3, 256), (5, 504), (4, 512), (7, 520), (130, 1368), (9, 2048), (6, 2056), (33, 4096), (2, 8200)]


def run(x, resid, gamma, beta, eps, y, dim, sum=None, stream=None):
    X.xema_op_layernorm(X.layernorm_args(x, CODE[x.dtype], x.shape[0], dim, gamma, beta, eps, y, CODE[y.dtype], resid=resid,
                                         resid_dtype=CODE[resid.dtype] if resid is not None else 0, sum=sum,
                                         sum_dtype=CODE[sum.dtype] if sum is not None else 0, ldx=ld(x),
                                         ld_resid=ld(resid) if resid is not None else 0, ld_sum=ld(sum) if sum is not None else 0, ldy=ld(y)), stream)


def run_bwd(s, dy, dsum, gamma, eps, dx, dgamma, dbeta, dim, stream=None):
    n = X.xema_layernorm_bwd_workspace_bytes(s.shape[0], dim)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)
    X.xema_op_layernorm_bwd(X.layernorm_bwd_args(s, CODE[s.dtype], s.shape[0], dim, gamma, eps, dy, CODE[dy.dtype], dx, CODE[dx.dtype], dgamma, dbeta,
                                                 ws, n, dsum=dsum, dsum_dtype=CODE[dsum.dtype] if dsum is not None else 0, ld_s=ld(s), ld_dy=ld(dy),
                                                 ld_dsum=ld(dsum) if dsum is not None else 0, ld_dx=ld(dx)), stream)


@pytest.mark.parametrize("rows,dim", SIZES)
@pytest.mark.parametrize("xt,rt,yt", [(BF16, None, BF16), (F16, F32, F16), (F32, F32, BF16), (BF16, BF16, F16), (F32, None, F32), (F16, F16, F32)])
def test_layernorm(rows, dim, xt, rt, yt):
    g = gen(rows * 7 + dim)
    x, _ = strided(normal(g, (rows, dim), 2.0, xt, 1.5), 8)
    resid = strided(normal(g, (rows, dim), 3.0, rt), 16)[0] if rt else None
    gamma = normal(g, (dim,), 0.3, mean=1.0) if dim % 16 or dim == 512 else None
    beta = normal(g, (dim,), 0.5) if dim % 16 or dim == 4096 else None
    y, s = empty(rows, dim, 24, yt), empty(rows, dim, 8, rt or F32)
    run(x, resid, gamma, beta, 1e-5, y, dim, s)
    want_s, want, err = R.layernorm(x, resid, gamma, beta, 1e-5)
    R.within(y[:, :dim], want, R.rounded(want, err, yt), "y")
    R.within(s[:, :dim], want_s, R.rounded(want_s, R.U * want_s.abs(), s.dtype), "sum")
    gap_kept(y, dim)
    gap_kept(s, dim)


@pytest.mark.parametrize("rows,dim", SIZES + [(4200, 264), (1500, 2200)])
@pytest.mark.parametrize("st,dt,at,ot", [(BF16, BF16, None, BF16), (F16, F32, F32, F32), (F32, F16, F16, F16), (F32, BF16, BF16, F32)])
def test_gradient(rows, dim, st, dt, at, ot):
    g = gen(rows + dim)
    s, dy = strided(normal(g, (rows, dim), 2.0, st, -0.7), 8)[0], strided(normal(g, (rows, dim), 0.5, dt, 0.1), 16)[0]
    dsum = strided(normal(g, (rows, dim), 0.3, at), 8)[0] if at else None
    gamma = normal(g, (dim,), 0.3, mean=1.0) if dim % 16 or dim == 512 else None
    dx, dgamma, dbeta = empty(rows, dim, 24, ot), torch.full((dim,), 7.0, device=DEV), torch.full((dim,), 7.0, device=DEV)
    run_bwd(s, dy, dsum, gamma, 1e-5, dx, dgamma, dbeta, dim)
    want = R.layernorm_bwd(s, dy, dsum, gamma, 1e-5)
    R.within(dx[:, :dim], want["dx"][0], R.rounded(*want["dx"], ot), "dx")
    R.within(dgamma, *want["dgamma"], "dgamma")
    R.within(dbeta, *want["dbeta"], "dbeta")
    gap_kept(dx, dim)
    # each output alone has the same bytes
    for dg, db in ((None, None), (dgamma, None), (None, dbeta)):
        kept = [t.clone() for t in (dx, dgamma, dbeta)]
        dx.view(torch.uint8).fill_(0xFF)
        run_bwd(s, dy, dsum, gamma, 1e-5, dx, dg, db, dim)
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(kept, (dx, dgamma, dbeta)))


@pytest.mark.parametrize("dim", [264, 520, 1032, 2056, 4104, 8200])
def test_every_type_at_every_width_of_waves(dim):
    """All types of every argument, for each number of waves that a row takes."""
    rows, types = 19, (BF16, F16, F32)
    g = gen(dim)
    gamma, beta = normal(g, (dim,), 0.3, mean=1.0), normal(g, (dim,), 0.3)
    s, dy, dsum = ({t: normal(g, (rows, dim), std, t, mean) for t in types} for std, mean in ((2.0, -0.7), (0.5, 0.1), (0.3, 0.0)))
    for st in types:
        for dt in types:
            for at in (None, *types):
                want = R.layernorm_bwd(s[st], dy[dt], dsum[at] if at else None, gamma, 1e-5)
                for ot in types:
                    dx, dg, db = empty(rows, dim, 0, ot), torch.full((dim,), 7.0, device=DEV), torch.full((dim,), 7.0, device=DEV)
                    run_bwd(s[st], dy[dt], dsum[at] if at else None, gamma, 1e-5, dx, dg, db, dim)
                    R.within(dx, want["dx"][0], R.rounded(*want["dx"], ot), ("dx", st, dt, at, ot))
                    R.within(dg, *want["dgamma"], ("dgamma", st, dt, at, ot))
                    R.within(db, *want["dbeta"], ("dbeta", st, dt, at, ot))
            for yt in types:
                for sumt in (None, *types):
                    y, total = empty(rows, dim, 0, yt), empty(rows, dim, 0, sumt) if sumt else None
                    for r in (None, dy[dt]):
                        run(s[st], r, gamma, beta, 1e-5, y, dim, total)
                        want_s, want, err = R.layernorm(s[st], r, gamma, beta, 1e-5)
                        R.within(y, want, R.rounded(want, err, yt), ("y", st, dt, yt))
                        if sumt:
                            R.within(total, want_s, R.rounded(want_s, R.U * want_s.abs(), sumt), ("sum", st, dt, sumt))


def test_gradient_against_differences():
    """The formula's own gradient in 64 bits meets central differences of sum(dy * y) + sum(dsum * s)."""
    g = gen(5)
    s, dy, dsum, gamma = (torch.randn(n, generator=g, device=DEV, dtype=torch.float64) for n in ((3, 24), (3, 24), (3, 24), (24,)))
    want = R.layernorm_bwd(s, dy, dsum, gamma, 1e-5)

    def loss():
        e = s - s.mean(1, keepdim=True)
        return float((dy * e / torch.sqrt((e * e).mean(1, keepdim=True) + 1e-5) * gamma).sum() + (dsum * s).sum())

    for t, name, at in ((s, "dx", (1, 3)), (s, "dx", (2, 23)), (gamma, "dgamma", (5,))):
        x, ends = float(t[at]), []
        for h in (1e-4, -1e-4):
            t[at] = x + h
            ends.append(loss())
        t[at] = x
        assert abs((ends[0] - ends[1]) / 2e-4 - float(want[name][0][at])) < 1e-5


@pytest.mark.parametrize("dim", [512, 4096])
def test_constant_rows_large_means_and_non_finite_rows(dim):
    g = gen(1)
    x = normal(g, (6, dim), 1.0, F32)
    x[1] = 3.0                       # no variance: beta alone
    x[2] += 4096.0                   # a mean far above the deviation: taken about the mean, its bits are kept
    x[3, 5] = float("inf")
    x[4, 7] = float("nan")
    beta = normal(g, (dim,))
    y = empty(6, dim, 0, F32)
    run(x, None, None, beta, 1e-6, y, dim)
    fine = [0, 1, 2, 5]
    _, want, err = R.layernorm(x[fine], None, None, beta, 1e-6)
    R.within(y[fine], want, R.rounded(want, err, F32), "finite rows")
    assert torch.equal(y[1], beta.float()) and bool(torch.isnan(y[3:5]).all())


def test_outputs_that_are_an_input():
    g = gen(2)
    x, resid, gamma = normal(g, (70, 520)), normal(g, (70, 520), 1.0, F32), normal(g, (520,), 0.2, mean=1.0)
    y, s = empty(70, 520, 0, BF16), empty(70, 520, 0, F32)
    run(x, resid, gamma, None, 1e-6, y, 520, s)
    y2, r2 = empty(70, 520, 0, BF16), resid.clone()
    run(x, r2, gamma, None, 1e-6, y2, 520, r2)
    assert torch.equal(y, y2) and torch.equal(r2, s)
    dy, dsum = normal(g, (70, 520)), normal(g, (70, 520))
    dx, dg, db = empty(70, 520, 0, BF16), torch.empty(520, device=DEV), torch.empty(520, device=DEV)
    run_bwd(x, dy, dsum, gamma, 1e-6, dx, dg, db, 520)
    for i in range(3):
        t = [x.clone(), dy.clone(), dsum.clone()]
        dg2, db2 = torch.empty(520, device=DEV), torch.empty(520, device=DEV)
        run_bwd(t[0], t[1], t[2], gamma, 1e-6, t[i], dg2, db2, 520)
        assert torch.equal(t[i], dx) and torch.equal(dg, dg2) and torch.equal(db, db2)


def test_no_rows():
    x, dg, db = torch.empty((8, 64), device=DEV, dtype=BF16), torch.full((64,), 7.0, device=DEV), torch.full((64,), 7.0, device=DEV)
    y = empty(8, 64, 0, BF16)
    X.xema_op_layernorm(X.layernorm_args(x, 0, 0, 64, None, None, 1e-6, y, 0))
    n = X.xema_layernorm_bwd_workspace_bytes(0, 64)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    X.xema_op_layernorm_bwd(X.layernorm_bwd_args(x, 0, 0, 64, None, 1e-6, x, 0, y, 0, dg, db, ws, n))
    assert bool((dg == 0).all()) and bool((db == 0).all())
    gap_kept(y, 0)
