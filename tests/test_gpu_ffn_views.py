"""Inputs and outputs that are column ranges of one buffer, or that are each
other where the header allows it: the same bytes as from tensors of their own,
and nothing written beside the output's columns."""
import pytest
import torch

import paper_2607_11136_amd as X
from test_gpu_ffn import BF16, CODE, DEV, F16, E4M3, empty, empty_pre, gen, lora_inputs, normal, run_bwd, run_gated, run_lora, run_norm, spread_ids

pytestmark = pytest.mark.gpu


class Buffer:
    """Rows of the columns of several 16-bit matrices, 8 elements between them and behind the last."""

    def __init__(self, rows, dtype, **widths):
        self.buf = torch.full((rows, sum(widths.values()) + 8 * len(widths)), 3.0, device=DEV, dtype=dtype)
        self.at, c = {}, 0
        for n, w in widths.items():
            self.at[n] = slice(c, c + w)
            c += w + 8

    def __getitem__(self, n):
        return self.buf[:, self.at[n]]

    def fill(self, n, t):
        self[n].copy_(t)
        return self[n]

    def others(self, n):
        keep = torch.ones(self.buf.shape[1], dtype=torch.bool, device=DEV)
        keep[self.at[n]] = False
        return self.buf[:, keep].clone()


@pytest.mark.parametrize("rows,dim,hidden", [(1, 64, 136), (20, 264, 392), (300, 136, 264), (2100, 512, 1032)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_outputs_beside_inputs(rows, dim, hidden, dtype):
    g = gen(rows)
    b = Buffer(rows, dtype, x=dim, h=dim, y=hidden, z=dim, dx=dim)
    x, gamma = b.fill("x", normal(g, (rows, dim), 1.0, dtype)), normal(g, (dim,), 0.2, mean=1.0)
    wg, wu = normal(g, (hidden, dim), dim ** -0.5, dtype), normal(g, (hidden, dim), dim ** -0.5, dtype)
    d = lora_inputs(rows, hidden, dim, 16, 3, dtype, rows)
    ids = spread_ids(rows, 3, "mixed", rows)

    def step(n, call, *own):
        """call() on the buffer's columns `n`, with everything else as it was."""
        before = b.others(n)
        call()
        assert torch.equal(before, b.others(n))
        for t in own:
            assert torch.equal(b[n].view(torch.int16), t.view(torch.int16)), n

    h = empty(rows, dim, 0, dtype)
    run_norm(x.contiguous(), None, gamma, 1e-6, h, dim)
    step("h", lambda: run_norm(x, None, gamma, 1e-6, b["h"], dim), h)
    y, pre, pre2 = empty(rows, hidden, 0, dtype), empty_pre(rows, hidden), empty_pre(rows, hidden)
    run_gated(h, wg, wu, None, None, 0, y, pre)
    step("y", lambda: run_gated(b["h"], wg, wu, None, None, 0, b["y"], pre2), y)
    assert torch.equal(pre, pre2)
    z, zeros = torch.zeros((rows, dim), device=DEV, dtype=dtype), b.fill("z", torch.zeros((rows, dim), device=DEV))
    run_lora({**d, "x": y}, ids, z)
    step("z", lambda: run_lora({**d, "x": b["y"]}, ids, zeros), z)
    want = run_bwd(h, wg, wu, pre, y, 0, gap=0)
    n = X.xema_gated_ffn_bwd_workspace_bytes(rows, dim, hidden)
    ws, dw = torch.empty(n, dtype=torch.uint8, device=DEV), [empty(hidden, dim, 0, dtype) for _ in range(2)]
    ld = b.buf.stride(0)
    step("dx", lambda: X.xema_op_gated_ffn_bwd(X.gated_ffn_bwd_args(CODE[dtype], 0, b["h"], rows, dim, wg, wu, hidden, pre, b["y"], b["dx"], dw[0], dw[1],
                                                                    ws, n, ldx=ld, ld_dy=ld, ld_dx=ld)), want["dx"])
    assert torch.equal(dw[0], want["dgate_w"]) and torch.equal(dw[1], want["dup_w"])
    dx = empty(rows, dim, 0, dtype)
    X.xema_op_rmsnorm_bwd(X.rmsnorm_bwd_args(x.contiguous(), CODE[dtype], rows, dim, gamma, 1e-6, want["dx"], CODE[dtype], dx, CODE[dtype]))
    step("z", lambda: X.xema_op_rmsnorm_bwd(X.rmsnorm_bwd_args(x, CODE[dtype], rows, dim, gamma, 1e-6, b["dx"], CODE[dtype], b["z"], CODE[dtype],
                                                               ld_s=ld, ld_dy=ld, ld_dx=ld)), dx)


def test_codes_beside_the_row():
    """e4m3 rows in the bytes behind each 16-bit row."""
    rows, dim = 130, 512
    x = normal(gen(1), (rows, dim))
    buf = torch.zeros((rows, 3 * dim + 16), dtype=torch.uint8, device=DEV)
    buf[:, :2 * dim] = x.view(torch.uint8)
    xv, yv = buf.view(torch.bfloat16)[:, :dim], buf.view(E4M3)[:, 2 * dim:3 * dim]
    want, ws, scale = empty(rows, dim, 0, E4M3), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    run_norm(x, None, None, 1e-6, want, dim, None, ws)
    run_norm(xv, None, None, 1e-6, yv, dim, None, scale)
    assert torch.equal(yv.view(torch.uint8), want.view(torch.uint8)) and torch.equal(ws, scale)
    assert torch.equal(buf[:, :2 * dim], x.view(torch.uint8)) and bool((buf[:, 3 * dim:] == 0).all())


@pytest.mark.parametrize("shift", [8, 64, -64])
def test_columns_that_do_overlap_are_refused(shift):
    buf = torch.zeros((40, 512), device=DEV, dtype=BF16)
    with pytest.raises(X.XemaError) as e:
        run_norm(buf[:, 128:256], None, None, 1e-6, buf[:, 128 + shift:256 + shift], 128)
    assert e.value.status == X.XEMA_ERR_INVALID_ARG


@pytest.mark.parametrize("rows,dim", [(5, 512), (130, 2064), (3, 16384)])
@pytest.mark.parametrize("dtype,other", [(BF16, None), (torch.float32, BF16), (F16, F16)])
@pytest.mark.parametrize("out", [F16, E4M3])
def test_the_sum_in_place_of_x(rows, dim, dtype, other, out):
    g = gen(dim)
    x, resid = normal(g, (rows, dim + 8), 1.0, dtype), normal(g, (rows, dim), 2.0, other) if other else None
    scales = [torch.empty(rows, device=DEV) if out == E4M3 else None for _ in range(2)]
    y, y2 = empty(rows, dim, 0, out), empty(rows, dim, 0, out)
    want, kept = empty(rows, dim, 0, dtype), x.clone()
    run_norm(kept[:, :dim], resid, None, 1e-6, y, dim, want, scales[0])
    run_norm(x[:, :dim], resid, None, 1e-6, y2, dim, x[:, :dim], scales[1])
    assert torch.equal(x[:, :dim], want) and torch.equal(x[:, dim:], kept[:, dim:]) and torch.equal(y.view(torch.uint8), y2.view(torch.uint8))
    assert out != E4M3 or torch.equal(*scales)


@pytest.mark.parametrize("rows,dim", [(5, 512), (5000, 264), (1030, 4096)])
def test_one_gradient_for_both_paths_in_place(rows, dim):
    """dy, dsum and dx one tensor: a row is read whole before it is written."""
    g = gen(rows)
    s, d, gamma = normal(g, (rows, dim)), normal(g, (rows, dim)), normal(g, (dim,), 0.2, mean=1.0)
    ws = [torch.empty(X.xema_rmsnorm_bwd_workspace_bytes(rows, dim), dtype=torch.uint8, device=DEV) for _ in range(2)]
    dg, dx = [torch.empty(dim, device=DEV) for _ in range(2)], empty(rows, dim, 0, BF16)
    X.xema_op_rmsnorm_bwd(X.rmsnorm_bwd_args(s, 0, rows, dim, gamma, 1e-6, d, 0, dx, 0, dg[0], ws[0], ws[0].numel(), dsum=d, dsum_dtype=0))
    X.xema_op_rmsnorm_bwd(X.rmsnorm_bwd_args(s, 0, rows, dim, gamma, 1e-6, d, 0, d, 0, dg[1], ws[1], ws[1].numel(), dsum=d, dsum_dtype=0))
    assert torch.equal(d, dx) and torch.equal(*dg)
