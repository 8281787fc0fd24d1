"""Every launch of a feed-forward entry point goes to the stream of its call:
the inputs arrive on that stream behind work that is still running when the
call returns, so a launch anywhere else meets what the buffers held before."""
import pytest
import torch

import paper_2607_11136_amd as X
from test_gpu_ffn import BF16, DEV, E4M3, F32, empty, empty_pre, gen, lora_inputs, normal, run_gated, run_norm, spread_ids

pytestmark = pytest.mark.gpu


def norm(rows, out):
    g = gen(1)
    x, resid, gamma = normal(g, (rows, 1024)), normal(g, (rows, 1024), 2.0, F32), normal(g, (1024,), 0.2, mean=1.0)
    y, s, scale = empty(rows, 1024, 0, out), empty(rows, 1024, 0, F32), torch.empty(rows, device=DEV)
    return [x, resid, gamma], [y, s] + [scale] * (out == E4M3), [], lambda st: run_norm(x, resid, gamma, 1e-6, y, 1024, s, scale if out == E4M3 else None, st)


def norm_bwd(rows):
    g = gen(2)
    s, dy, gamma = normal(g, (rows, 1024)), normal(g, (rows, 1024)), normal(g, (1024,), 0.2, mean=1.0)
    dx, dgamma = empty(rows, 1024, 0, BF16), empty(1, 1024, 0, F32)[0]
    ws = torch.empty(X.xema_rmsnorm_bwd_workspace_bytes(rows, 1024), dtype=torch.uint8, device=DEV)
    a = X.rmsnorm_bwd_args(s, 0, rows, 1024, gamma, 1e-6, dy, 0, dx, 0, dgamma, ws, ws.numel())
    return [s, dy, gamma], [dx, dgamma], [ws], lambda st: X.xema_op_rmsnorm_bwd(a, st)


def gated(rows):
    g = gen(3)
    x, wg, wu = normal(g, (rows, 264)), normal(g, (520, 264), 0.06), normal(g, (520, 264), 0.06)
    y, pre = empty(rows, 520, 0, BF16), empty_pre(rows, 520)
    return [x, wg, wu], [y, pre], [], lambda st: run_gated(x, wg, wu, None, None, 1, y, pre, st)


def gated_bwd(rows, dim, hidden):
    g = gen(4)
    x, wg, wu, dy = normal(g, (rows, dim)), normal(g, (hidden, dim), 0.06), normal(g, (hidden, dim), 0.06), normal(g, (rows, hidden))
    pre = empty_pre(rows, hidden)
    run_gated(x, wg, wu, None, None, 0, empty(rows, hidden, 0, BF16), pre)
    out = [empty(rows, dim, 0, BF16), empty(hidden, dim, 0, BF16), empty(hidden, dim, 0, BF16), empty(1, hidden, 0, BF16)[0], empty(1, hidden, 0, BF16)[0]]
    ws = torch.empty(X.xema_gated_ffn_bwd_workspace_bytes(rows, dim, hidden), dtype=torch.uint8, device=DEV)
    a = X.gated_ffn_bwd_args(0, 0, x, rows, dim, wg, wu, hidden, pre, dy, out[0], out[1], out[2], ws, ws.numel(), dgate_b=out[3], dup_b=out[4])
    return [x, wg, wu, dy, pre], out, [ws], lambda st: X.xema_op_gated_ffn_bwd(a, st)


def lora(rows):
    d, ids = lora_inputs(rows, 264, 392, 16, 3, BF16, 5), spread_ids(rows, 3, "one", 5)
    x, y = d["x"].contiguous(), empty(rows, 392, 0, BF16)
    ws = torch.empty(X.xema_lora_workspace_bytes(rows, 16), dtype=torch.uint8, device=DEV)
    a = X.lora_args(0, x, rows, 264, d["w"], 392, d["bias"], d["a"], d["b"], d["scale"], 16, 3, ids, y, 0, ws, ws.numel())
    return [x, d["w"], d["bias"], d["a"], d["b"], d["scale"], ids], [y], [ws], lambda st: X.xema_op_lora_linear(a, st)


CASES = {
    "norm": lambda: norm(300, BF16), "norm 8 bits": lambda: norm(300, E4M3), "norm gradient": lambda: norm_bwd(3000),
    "gated, few rows": lambda: gated(7), "gated": lambda: gated(700),
    "gated gradient, one launch of products": lambda: gated_bwd(65, 136, 200), "two launches": lambda: gated_bwd(1614, 1240, 2400),
    "split dx": lambda: gated_bwd(70, 136, 4104), "split weights' gradients": lambda: gated_bwd(4500, 64, 72),
    "projection, few rows": lambda: lora(20), "projection, reduction by rows": lambda: lora(300), "projection": lambda: lora(2100),
}


@pytest.mark.parametrize("how", ["stream argument", "current stream"])
@pytest.mark.parametrize("case", CASES)
def test_launches_follow_the_work_of_their_stream(case, how):
    inputs, outputs, scratch, call = CASES[case]()
    call(None)
    torch.cuda.synchronize()
    want, real = [t.clone() for t in outputs], [t.clone() for t in inputs]
    long = torch.ones((8192, 8192), device=DEV, dtype=BF16)
    torch.mm(long, long)
    s = torch.cuda.Stream()
    for products in (200, 1000, 4000):        # (more where the host was slow, or the call would prove nothing)
        # NaN in every type, and rows without an adapter: any launch that does not wait leaves its mark
        for t in inputs:
            t.view(torch.uint8).fill_(0xFF) if t.dtype != torch.int32 else t.fill_(-1)
        for t in (*outputs, *scratch):
            t.view(torch.uint8).fill_(0xFF)
        torch.cuda.synchronize()
        reached = torch.cuda.Event()
        with torch.cuda.stream(s):
            for _ in range(products):
                torch.mm(long, long)
            for t, r in zip(inputs, real):
                t.copy_(r)
            reached.record()
            if how == "current stream":
                call(None)
        if how == "stream argument":
            call(s)
        running = not reached.query()
        with torch.cuda.stream(s):
            got = [t.clone() for t in outputs]
        s.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(g.view(torch.uint8), w.view(torch.uint8)), case
        if running:
            return
    raise AssertionError("the work was always done before the call returned")


def test_the_marks_are_seen():
    """Run on the inputs that a launch on another stream would meet, every case gives other bytes."""
    for case, make in CASES.items():
        inputs, outputs, _, call = make()
        call(None)
        want = [t.clone() for t in outputs]
        for t in inputs:
            t.view(torch.uint8).fill_(0xFF) if t.dtype != torch.int32 else t.fill_(-1)
        call(None)
        torch.cuda.synchronize()
        assert any(not torch.equal(t.view(torch.uint8), w.view(torch.uint8)) for t, w in zip(outputs, want)), case


@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("handle", [0, 1, 2])
def test_handles_of_implicit_streams(case, handle):
    """NULL, hipStreamLegacy and hipStreamPerThread."""
    inputs, outputs, _, call = CASES[case]()
    call(None)
    torch.cuda.synchronize()
    want = [t.clone() for t in outputs]
    for t in outputs:
        t.view(torch.uint8).fill_(0xFF)
    torch.cuda.synchronize()
    call(handle)
    torch.cuda.synchronize()
    assert all(torch.equal(t.view(torch.uint8), w.view(torch.uint8)) for t, w in zip(outputs, want))
