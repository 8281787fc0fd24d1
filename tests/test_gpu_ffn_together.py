"""The feed-forward operators as a program uses them: a sub-block served in 16
and in 8 bits with adapters, a training step down to the norm's gradient; the
same captured into a graph and replayed, on other streams, two at once, and at
offsets past 32 bits."""
import pytest
import torch

import ffn_reference as R
import paper_2607_11136_amd as X
from test_gpu_ffn import (BF16, CODE, DEV, E4M3, F16, F32, check_e4m3, empty, empty_pre, gen, lora_inputs, normal, run_bwd, run_gated, run_lora,
                          run_norm, spread_ids)

pytestmark = pytest.mark.gpu


class SubBlock:
    """x + resid -> norm -> gated -> down projection with adapters, the buffers allocated once."""

    def __init__(self, rows, dim, hidden, dtype, eight_bit, seed):
        g = gen(seed)
        self.rows, self.dim, self.hidden, self.dtype, self.eight_bit = rows, dim, hidden, dtype, eight_bit
        self.x, self.resid = normal(g, (rows, dim), 1.0, dtype), normal(g, (rows, dim), 1.5, F32)
        self.gamma = normal(g, (dim,), 0.2, mean=1.0)
        w = [normal(g, (hidden, dim), dim ** -0.5, F32) for _ in range(2)]
        if eight_bit:
            self.scales = [t.abs().amax(1) / 448 for t in w]
            self.w = [(t / s[:, None]).to(E4M3) for t, s in zip(w, self.scales)]
            self.h, self.h_scale = empty(rows, dim, 0, E4M3), torch.empty(rows, device=DEV)
        else:
            self.scales, self.w = [None, None], [t.to(dtype) for t in w]
            self.h, self.h_scale = empty(rows, dim, 0, dtype), None
        self.lora = lora_inputs(rows, hidden, dim, 16, 3, dtype, seed + 1)
        self.ids = spread_ids(rows, 3, "runs", seed)
        self.sum, self.g, self.y = empty(rows, dim, 0, F32), empty(rows, hidden, 0, dtype), empty(rows, dim, 0, dtype)
        self.ws = torch.empty(X.xema_lora_workspace_bytes(rows, 16), dtype=torch.uint8, device=DEV)

    def run(self, stream=None):
        c = CODE[self.dtype]
        run_norm(self.x, self.resid, self.gamma, 1e-6, self.h, self.dim, self.sum, self.h_scale, stream)
        X.xema_op_gated_ffn(X.gated_ffn_args(CODE[self.h.dtype], 0, self.h, self.rows, self.dim, self.w[0], self.w[1], self.hidden, self.g, c,
                                             x_scale=self.h_scale, gate_scale=self.scales[0], up_scale=self.scales[1]), stream)
        d = self.lora
        X.xema_op_lora_linear(X.lora_args(c, self.g, self.rows, self.hidden, d["w"], self.dim, d["bias"], d["a"], d["b"], d["scale"], 16, 3,
                                          self.ids, self.y, c, self.ws, self.ws.numel()), stream)

    def outputs(self):
        return [t for t in (self.sum, self.h, self.h_scale, self.g, self.y) if t is not None]

    def check(self):
        """Each stage against its definition, given what the one before stored."""
        s, h, rel = R.rmsnorm(self.x, self.resid, self.gamma, 1e-6)
        R.within(self.sum, s, R.rounded(s, R.U * s.abs(), F32), "sum")
        stored = self.h.double()
        if self.eight_bit:
            check_e4m3(self.h, self.h_scale, h, rel, "h")
            stored = stored * self.h_scale.double()[:, None]
            w = [t.double() * sc.double()[:, None] for t, sc in zip(self.w, self.scales)]
        else:
            R.within(self.h, h, R.rounded(h, rel * h.abs(), self.dtype), "h")
            w = self.w
        g, e, *_ = R.gated(stored, w[0], w[1], None, None, 0, slack=2.0 ** -14 if self.eight_bit else 0.0)
        R.within(self.g, g, R.rounded(g, e, self.dtype), "g")
        d = self.lora
        y, e = R.lora(self.g, d["w"], d["bias"], d["a"], d["b"], d["scale"], self.ids, self.dtype)
        live = self.ids >= -1
        R.within(self.y[live], y[live], R.rounded(y, e, self.dtype)[live], "y")
        assert bool((self.y[~live].view(torch.int16) == -1).all())


@pytest.mark.parametrize("rows,dim,hidden", [(1, 512, 1024), (40, 1040, 2064), (700, 528, 1376), (2300, 1024, 4096)])
@pytest.mark.parametrize("dtype,eight_bit", [(BF16, False), (F16, False), (BF16, True)])
def test_sub_block(rows, dim, hidden, dtype, eight_bit):
    b = SubBlock(rows, dim, hidden, dtype, eight_bit, rows)
    b.run()
    b.check()


@pytest.mark.parametrize("rows,eight_bit", [(1, False), (33, True), (515, False), (2300, True)])
def test_sub_block_in_a_graph(rows, eight_bit):
    """Captured once, replayed on inputs that change between the replays, with
    eager work on the same buffers between them; every replay has the eager bytes."""
    b = SubBlock(rows, 528, 1376, BF16, eight_bit, rows)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        b.run()
    for turn in range(4):
        b.x.copy_(normal(gen(100 + turn), b.x.shape))
        b.ids.copy_(spread_ids(rows, 3, ("mixed", "one", "runs", "mixed")[turn], turn))
        for t in b.outputs():
            t.view(torch.uint8).fill_(0xFF)
        b.run()
        torch.cuda.synchronize()
        want = [t.clone() for t in b.outputs()]
        for t in b.outputs():
            t.view(torch.uint8).fill_(0xFF)
        b.ws.fill_(0xAA)
        graph.replay()
        torch.cuda.synchronize()
        for w, t in zip(want, b.outputs()):
            assert torch.equal(w.view(torch.uint8), t.view(torch.uint8)), turn


def test_training_step_in_a_graph_and_on_two_streams():
    rows, dim, hidden = 300, 264, 520
    g = gen(7)
    w = [normal(g, (hidden, dim), dim ** -0.5) for _ in range(2)]
    wss = [torch.empty(X.xema_gated_ffn_bwd_workspace_bytes(rows, dim, hidden), dtype=torch.uint8, device=DEV) for _ in range(2)]
    wsn = [torch.empty(X.xema_rmsnorm_bwd_workspace_bytes(rows, dim), dtype=torch.uint8, device=DEV) for _ in range(2)]
    gamma = normal(g, (dim,), 0.2, mean=1.0)
    xs, dys = [normal(g, (rows, dim)) for _ in range(2)], [normal(g, (rows, hidden)) for _ in range(2)]
    outs = [{"h": empty(rows, dim, 0, BF16), "y": empty(rows, hidden, 0, BF16), "pre": empty_pre(rows, hidden), "dh": empty(rows, dim, 0, BF16),
             "dg": empty(hidden, dim, 0, BF16), "du": empty(hidden, dim, 0, BF16), "bg": empty(1, hidden, 0, BF16)[0],
             "bu": empty(1, hidden, 0, BF16)[0], "dx": empty(rows, dim, 0, BF16), "dgamma": empty(1, dim, 0, F32)[0]} for _ in range(2)]

    def step(i, stream=None):
        o = outs[i]
        run_norm(xs[i], None, gamma, 1e-6, o["h"], dim, stream=stream)
        run_gated(o["h"], w[0], w[1], None, None, 1, o["y"], o["pre"], stream)
        X.xema_op_gated_ffn_bwd(X.gated_ffn_bwd_args(0, 1, o["h"], rows, dim, w[0], w[1], hidden, o["pre"], dys[i], o["dh"], o["dg"], o["du"],
                                                     wss[i], wss[i].numel(), dgate_b=o["bg"], dup_b=o["bu"]), stream)
        X.xema_op_rmsnorm_bwd(X.rmsnorm_bwd_args(xs[i], 0, rows, dim, gamma, 1e-6, o["dh"], 0, o["dx"], 0, o["dgamma"], wsn[i], wsn[i].numel(),
                                                 dsum=o["dh"], dsum_dtype=0), stream)

    def poison():
        for o in outs:
            for t in o.values():
                t.view(torch.uint8).fill_(0xFF)
        for t in (*wss, *wsn):
            t.fill_(0xFF)
        torch.cuda.synchronize()

    for i in range(2):
        step(i)
    torch.cuda.synchronize()
    want = [{n: t.clone() for n, t in o.items()} for o in outs]
    o = want[0]
    ref = R.rmsnorm_bwd(xs[0], o["dh"], o["dh"], gamma, 1e-6)
    R.within(o["dx"], ref["dx"][0], R.rounded(ref["dx"][0], ref["dx"][1], BF16), "dx")
    R.within(o["dgamma"], *ref["dgamma"], "dgamma")
    same = lambda: all(torch.equal(t.view(torch.uint8), w_[n].view(torch.uint8)) for o_, w_ in zip(outs, want) for n, t in o_.items())  # noqa: E731
    # two steps at once, on streams of their own
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        poison()
        step(0, a)
        step(1, b)
        torch.cuda.synchronize()
        assert same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=a):
        step(0)
        step(1)
    for _ in range(3):
        poison()
        graph.replay()
        torch.cuda.synchronize()
        assert same()
        step(1)


def test_streams_are_those_of_the_call():
    """Work goes to the stream of the call, after what that stream has queued."""
    x = torch.zeros((4000, 1024), device=DEV, dtype=BF16)
    y = empty(4000, 1024, 0, BF16)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for i in range(200):
            x.add_(1)
        run_norm(x, None, None, 1e-6, y, 1024)
    s.synchronize()
    assert bool((y == 1).all())


def test_same_call_gives_the_same_bytes():
    b = SubBlock(1500, 1032, 4104, F16, False, 3)
    b.run()
    torch.cuda.synchronize()
    want = [t.clone() for t in b.outputs()]
    for _ in range(3):
        b.ws.fill_(0x55)
        b.run()
        torch.cuda.synchronize()
        assert all(torch.equal(w.view(torch.uint8), t.view(torch.uint8)) for w, t in zip(want, b.outputs()))


# -- offsets past 2^31 elements and 2^32 bytes ---------------------------------------------------------------------


def far_rows(rows, ld, width, dtype, seed, filled):
    """A [rows, width] view of rows `ld` apart: random in the last `filled` rows and the first, zeros between."""
    buf = torch.zeros((rows, ld), dtype=dtype, device=DEV)
    g = gen(seed)
    buf[0, :width] = normal(g, (width,), 1.0, dtype)
    buf[-filled:, :width] = normal(g, (filled, width), 1.0, dtype)
    return buf[:, :width]


ROWS, LD, LAST = 140000, 16392, 300      # 140000 * 16392 = 2.29e9 elements


def test_far_offsets_norm():
    x = far_rows(ROWS, LD, 64, BF16, 1, LAST)
    y = torch.empty((ROWS, LD), dtype=BF16, device=DEV)[:, :64]
    run_norm(x, None, None, 1e-6, y, 64)
    for part in (slice(0, 1), slice(ROWS - LAST, ROWS)):
        _, want, rel = R.rmsnorm(x[part], None, None, 1e-6)
        R.within(y[part], want, R.rounded(want, rel * want.abs(), BF16), "y")
    assert bool((y[1:1000] == 0).all())
    dgamma, n = torch.empty(64, device=DEV), X.xema_rmsnorm_bwd_workspace_bytes(ROWS, 64)
    dy, ws = y, torch.empty(n, dtype=torch.uint8, device=DEV)
    dx = torch.empty((ROWS, LD), dtype=BF16, device=DEV)[:, :64]
    X.xema_op_rmsnorm_bwd(X.rmsnorm_bwd_args(x, 0, ROWS, 64, None, 1e-6, dy, 0, dx, 0, dgamma, ws, n, ld_s=LD, ld_dy=LD, ld_dx=LD))
    part = torch.cat((torch.arange(1), torch.arange(ROWS - LAST, ROWS))).to(DEV)
    want = R.rmsnorm_bwd(x[part], dy[part], None, None, 1e-6)
    R.within(dx[part], want["dx"][0], R.rounded(want["dx"][0], want["dx"][1], BF16), "dx")
    R.within(dgamma, want["dgamma"][0], want["dgamma"][1], "dgamma")      # (the rows between add zeros)


@pytest.mark.parametrize("hidden", [72, 8200])
def test_far_offsets_gated(hidden):
    """Far x and y rows; with hidden 8200 y, pre and dg pass 2^31 bytes themselves."""
    x = far_rows(ROWS, LD if hidden == 72 else 64, 64, BF16, 2, LAST)
    g = gen(3)
    wg, wu = normal(g, (hidden, 64), 0.125), normal(g, (hidden, 64), 0.125)
    y = torch.empty((ROWS, LD if hidden == 72 else hidden), dtype=BF16, device=DEV)[:, :hidden]
    pre = torch.empty((ROWS, 6 * hidden), dtype=torch.uint8, device=DEV)
    run_gated(x, wg, wu, None, None, 0, y, pre)
    part = torch.cat((torch.arange(1), torch.arange(ROWS - LAST, ROWS))).to(DEV)
    want, e, *_ = R.gated(x[part], wg, wu, None, None, 0)
    R.within(y[part], want, R.rounded(want, e, BF16), "y")
    dy = y
    out = run_bwd(x, wg, wu, pre, dy, 0)
    from test_gpu_ffn import unpack24
    ref = R.gated_bwd(x[part], wg, wu, unpack24(pre[part].contiguous(), hidden), dy[part].contiguous(), 0, BF16)
    R.within(out["dx"][part][:, :64], ref["dx"][0], R.rounded(ref["dx"][0], ref["dx"][1], BF16), "dx")
    for n in ("dgate_w", "dup_w", "dgate_b", "dup_b"):
        R.within(out[n], ref[n][0], R.rounded(ref[n][0], ref[n][1], BF16), n)


def test_far_offsets_lora():
    d = lora_inputs(16, 64, 72, 8, 3, BF16, 5)
    d["x"] = far_rows(ROWS, LD, 64, BF16, 4, LAST)
    ids = torch.full((ROWS,), -2, dtype=torch.int32, device=DEV)
    ids[0], ids[-LAST:] = 1, torch.arange(LAST, device=DEV, dtype=torch.int32) // 120
    y = torch.empty((ROWS, LD), dtype=BF16, device=DEV)[:, :72]
    run_lora(d, ids, y)
    part = torch.cat((torch.arange(1), torch.arange(ROWS - LAST, ROWS))).to(DEV)
    want, e = R.lora(d["x"][part], d["w"], d["bias"], d["a"], d["b"], d["scale"], ids[part], BF16)
    R.within(y[part], want, R.rounded(want, e, BF16), "y")
