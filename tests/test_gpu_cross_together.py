"""The cross-attention operators as a program uses them: a sub-block served with
prompts of unlike length and its training step down to the norm's gradient; the
same captured into a graph and replayed, two at once on streams of their own,
behind work that still runs on their stream, and at offsets past 32 bits."""
import pytest
import torch

import cross_reference as R
import paper_2607_11136_amd as X
from test_gpu_cross_attn import Call
from test_gpu_ffn import BF16, CODE, DEV, F16, F32, empty, gen, normal
from test_gpu_layernorm import run as run_norm
from test_gpu_layernorm import run_bwd as run_norm_bwd
from test_gpu_linear import run as run_linear
from test_gpu_linear import run_bwd as run_linear_bwd

pytestmark = pytest.mark.gpu


class SubBlock:
    """x <- x + W_o Attn(W_q LayerNorm(x), W_kv e) + b_o, and its gradient; buffers allocated once."""

    def __init__(self, batch, heads, kv_heads, d, q_len, kv_len, enc, dtype, lens, seed):
        g = gen(seed)
        self.sizes, self.dtype, self.enc = (batch, heads, kv_heads, d, q_len, kv_len), dtype, enc
        D, nk, M, S = heads * d, kv_heads * d, batch * q_len, batch * kv_len
        self.D, self.nk = D, nk
        self.x, self.e = normal(g, (M, D), 1.5, F32), normal(g, (S, enc), 1.0, dtype)
        self.gamma, self.beta = normal(g, (D,), 0.2, mean=1.0), normal(g, (D,), 0.1)
        self.wq, self.wkv, self.wo = (normal(g, s, s[1] ** -0.5, dtype) for s in ((D, D), (2 * nk, enc), (D, D)))
        self.bq, self.bkv, self.bo = (normal(g, (n,), 0.2) for n in (D, 2 * nk, D))
        self.lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
        self.dy = normal(g, (M, D), 0.1, F32)
        t = dtype
        self.h, self.q, self.kv, self.o, self.y = (empty(M, D, 0, t), empty(M, D, 0, t), empty(S, 2 * nk, 0, t), empty(M, D, 0, t), empty(M, D, 0, F32))
        self.lse = torch.empty((batch, heads, q_len), device=DEV)
        self.do, self.dq, self.dkv, self.dh, self.de, self.dx = (empty(M, D, 0, t), empty(M, D, 0, t), empty(S, 2 * nk, 0, t), empty(M, D, 0, t),
                                                                  empty(S, enc, 0, t), empty(M, D, 0, F32))
        self.dwq, self.dwkv, self.dwo = (empty(*w.shape, 0, t) for w in (self.wq, self.wkv, self.wo))
        self.dbq, self.dbkv, self.dbo = (empty(1, b.numel(), 0, BF16)[0] for b in (self.bq, self.bkv, self.bo))
        self.dgamma, self.dbeta = torch.empty(D, device=DEV), torch.empty(D, device=DEV)
        sizes = [X.xema_cross_attn_workspace_bytes(*self.sizes), X.xema_cross_attn_bwd_workspace_bytes(*self.sizes)]
        sizes += [X.xema_linear_bwd_workspace_bytes(*s) for s in ((M, D, D), (S, enc, 2 * nk))] + [X.xema_layernorm_bwd_workspace_bytes(M, D), 256]
        self.ws = torch.empty(max(sizes), dtype=torch.uint8, device=DEV)

    def forward(self, stream=None):
        c, n = CODE[self.dtype], 2 * self.nk
        run_norm(self.x, None, self.gamma, self.beta, 1e-6, self.h, self.D, stream=stream)
        run_linear(self.h, self.wq, self.bq, 2, self.q, stream=stream)
        run_linear(self.e, self.wkv, self.bkv, 2, self.kv, stream=stream)
        X.xema_op_cross_attn(X.cross_attn_args(c, *self.sizes, self.q, self.kv, self.kv[:, self.nk:], self.sizes[3] ** -0.5, self.o, self.ws,
                                               self.ws.numel(), lse=self.lse, kv_lens=self.lens, ldk=n, ldv=n), stream)
        run_linear(self.o, self.wo, self.bo, 2, self.y, self.x, stream=stream)

    def backward(self, stream=None):
        c, n = CODE[self.dtype], 2 * self.nk
        run_linear_bwd(self.o, self.wo, None, self.dy, 2, self.do, self.dwo, self.dbo, stream, self.ws)
        X.xema_op_cross_attn_bwd(X.cross_attn_bwd_args(c, *self.sizes, self.q, self.kv, self.kv[:, self.nk:], self.sizes[3] ** -0.5, self.o, self.lse,
                                                       self.do, self.dq, self.dkv, self.dkv[:, self.nk:], self.ws, self.ws.numel(),
                                                       kv_lens=self.lens, ldk=n, ldv=n, ld_dk=n, ld_dv=n), stream)
        run_linear_bwd(self.e, self.wkv, None, self.dkv, 2, self.de, self.dwkv, self.dbkv, stream, self.ws)
        run_linear_bwd(self.h, self.wq, None, self.dq, 2, self.dh, self.dwq, self.dbq, stream, self.ws)
        X.xema_op_layernorm_bwd(X.layernorm_bwd_args(self.x, 2, self.x.shape[0], self.D, self.gamma, 1e-6, self.dh, c, self.dx, 2, self.dgamma,
                                                     self.dbeta, self.ws, self.ws.numel(), dsum=self.dy, dsum_dtype=2), stream)

    def step(self, stream=None):
        self.forward(stream)
        self.backward(stream)

    def outputs(self):
        return [self.h, self.q, self.kv, self.o, self.lse, self.y, self.do, self.dq, self.dkv, self.de, self.dh, self.dx, self.dwq, self.dwkv,
                self.dwo, self.dbq, self.dbkv, self.dbo, self.dgamma, self.dbeta]

    def poison(self):
        for t in (*self.outputs(), self.ws):
            t.view(torch.uint8).fill_(0xFF)
        torch.cuda.synchronize()

    def check(self):
        """Each stage against its definition, given what the one before stored."""
        b, h, kh, d, _, _ = self.sizes
        t = self.dtype

        def near(got, ref, kind, what):
            R.within(got, ref[0], R.rounded(*ref, kind) if kind else ref[1], what)

        near(self.h, R.layernorm(self.x, None, self.gamma, self.beta, 1e-6)[1:], t, "h")
        for got, x, w, bias, resid, kind in ((self.q, self.h, self.wq, self.bq, None, t), (self.kv, self.e, self.wkv, self.bkv, None, t),
                                             (self.y, self.o, self.wo, self.bo, self.x, F32)):
            near(got, R.linear(x, w, bias, 2, resid)[2:], kind, "projection")
        k, v, scale = self.kv[:, :self.nk], self.kv[:, self.nk:], d ** -0.5
        near(self.o, R.attention(self.q, k, v, b, h, kh, d, self.lens, scale, t)["o"], t, "o")
        for x, w, dy, got in ((self.o, self.wo, self.dy, (self.do, self.dwo, self.dbo)), (self.e, self.wkv, self.dkv, (self.de, self.dwkv, self.dbkv)),
                              (self.h, self.wq, self.dq, (self.dh, self.dwq, self.dbq))):
            ref = R.linear_bwd(x, w, None, dy, 2, t)
            for g_, n in zip(got, ("dx", "dw", "dbias")):
                near(g_, ref[n], t if n != "dbias" else BF16, n)
        ref = R.attention_bwd(self.q, k, v, self.o, self.lse, self.do, b, h, kh, d, self.lens, scale, t)
        for n, got in (("dq", self.dq), ("dk", self.dkv[:, :self.nk]), ("dv", self.dkv[:, self.nk:])):
            near(got, ref[n], t, n)
        ref = R.layernorm_bwd(self.x, self.dh, self.dy, self.gamma, 1e-6)
        near(self.dx, ref["dx"], F32, "dx")
        near(self.dgamma, ref["dgamma"], None, "dgamma")
        near(self.dbeta, ref["dbeta"], None, "dbeta")


BLOCKS = [((2, 4, 4, 64, 150, 77), 264, [77, 20]), ((3, 8, 2, 72, 40, 130), 136, [130, 0, 64]), ((1, 2, 2, 128, 700, 300), 520, [300]),
          ((4, 8, 1, 64, 1, 600), 72, [600, 599, 1, 33])]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("block", BLOCKS, ids=lambda b: str(b[0]))
def test_sub_block_and_its_gradient(block, dtype):
    b = SubBlock(*block[0], block[1], dtype, block[2], 1)
    b.poison()
    b.step()
    b.check()


@pytest.mark.parametrize("block", BLOCKS, ids=lambda b: str(b[0]))
def test_step_in_a_graph(block):
    """Captured once, replayed on inputs and lengths that change between the replays, with eager work on the same
    buffers between them; every replay has the eager bytes."""
    b = SubBlock(*block[0], block[1], BF16, block[2], 2)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        b.step()
    for turn in range(4):
        b.x.copy_(normal(gen(100 + turn), b.x.shape, 1.0, F32))
        b.lens.copy_(torch.randint(0, b.sizes[5] + 1, b.lens.shape, generator=gen(turn), device=DEV, dtype=torch.int32))
        b.poison()
        b.step()
        torch.cuda.synchronize()
        want = [t.clone() for t in b.outputs()]
        b.poison()
        graph.replay()
        torch.cuda.synchronize()
        for w, t in zip(want, b.outputs()):
            assert torch.equal(w.view(torch.uint8), t.view(torch.uint8)), turn


def test_two_steps_at_once():
    blocks = [SubBlock(*BLOCKS[i][0], BLOCKS[i][1], BF16, BLOCKS[i][2], 3 + i) for i in range(2)]
    for b in blocks:
        b.step()
    torch.cuda.synchronize()
    want = [[t.clone() for t in b.outputs()] for b in blocks]
    streams = [torch.cuda.Stream() for _ in blocks]
    for _ in range(3):
        for b in blocks:
            b.poison()
        for b, s in zip(blocks, streams):
            b.step(s)
        torch.cuda.synchronize()
        for b, w in zip(blocks, want):
            assert all(torch.equal(t.view(torch.uint8), x.view(torch.uint8)) for t, x in zip(b.outputs(), w))


# -- launches behind the work of their stream ----------------------------------------------------------------------


def attention(*size):
    c = Call(*size, BF16, [size[5] - 1] * size[0], seed=9, gap=0)
    return [c.q, c.kv, c.lens], [c.o, c.lse], [c.ws], c.forward


def attention_gradient(*size):
    c = Call(*size, BF16, [size[5] - 1] * size[0], seed=9, gap=0)
    c.forward()
    return [c.q, c.kv, c.do, c.lens], [c.dq, c.dkv], [c.ws], c.backward


def norm(rows):
    g = gen(1)
    x, resid, gamma, beta = normal(g, (rows, 1024)), normal(g, (rows, 1024), 2.0, F32), normal(g, (1024,), 0.2, mean=1.0), normal(g, (1024,))
    y, s = empty(rows, 1024, 0, BF16), empty(rows, 1024, 0, F32)
    return [x, resid, gamma, beta], [y, s], [], lambda st: run_norm(x, resid, gamma, beta, 1e-6, y, 1024, s, st)


def norm_bwd(rows):
    g = gen(2)
    s, dy, gamma = normal(g, (rows, 1024)), normal(g, (rows, 1024)), normal(g, (1024,), 0.2, mean=1.0)
    dx, dgamma, dbeta = empty(rows, 1024, 0, BF16), empty(1, 1024, 0, F32)[0], empty(1, 1024, 0, F32)[0]
    ws = torch.empty(X.xema_layernorm_bwd_workspace_bytes(rows, 1024), dtype=torch.uint8, device=DEV)
    a = X.layernorm_bwd_args(s, 0, rows, 1024, gamma, 1e-6, dy, 0, dx, 0, dgamma, dbeta, ws, ws.numel())
    return [s, dy, gamma], [dx, dgamma, dbeta], [ws], lambda st: X.xema_op_layernorm_bwd(a, st)


def linear(rows, out, dim=264):
    g = gen(3)
    x, w, r = normal(g, (rows, dim)), normal(g, (out, dim), 0.06), normal(g, (rows, out))
    y = empty(rows, out, 0, BF16)
    return [x, w, r], [y], [], lambda st: run_linear(x, w, None, 1, y, r, None, st)


def linear_bwd(rows, dim, out):
    g = gen(4)
    x, w, dy = normal(g, (rows, dim)), normal(g, (out, dim), 0.06), normal(g, (rows, out))
    pre = torch.empty(X.xema_linear_pre_bytes(rows, out), dtype=torch.uint8, device=DEV)
    run_linear(x, w, None, 0, empty(rows, out, 0, BF16), None, pre)
    o = [empty(rows, dim, 0, BF16), empty(out, dim, 0, BF16), empty(1, out, 0, BF16)[0]]
    ws = torch.empty(X.xema_linear_bwd_workspace_bytes(rows, dim, out), dtype=torch.uint8, device=DEV)
    return [x, w, dy, pre], o, [ws], lambda st: run_linear_bwd(x, w, pre, dy, 0, *o, st, ws)


CASES = {
    "attention": lambda: attention(1, 4, 4, 64, 700, 300), "attention in parts": lambda: attention(1, 2, 2, 128, 200, 2000),
    "single tokens": lambda: attention(130, 4, 2, 64, 1, 40), "single tokens in parts": lambda: attention(2, 8, 2, 128, 1, 3000),
    "attention gradient": lambda: attention_gradient(8, 40, 40, 64, 90, 40), "attention gradient in parts": lambda: attention_gradient(1, 3, 3, 72, 300, 1100),
    "norm": lambda: norm(300), "norm gradient": lambda: norm_bwd(3000), "linear, few rows": lambda: linear(7, 520), "linear": lambda: linear(700, 520),
    "linear, two launches": lambda: linear(9000, 2056, 520), "linear gradient, one launch of products": lambda: linear_bwd(65, 136, 200),
    "two launches": lambda: linear_bwd(3000, 1032, 4104), "split dx": lambda: linear_bwd(70, 136, 8200), "split dw": lambda: linear_bwd(4500, 64, 72),
}


def fill(t):
    t.view(torch.uint8).fill_(0xFF) if t.dtype != torch.int32 else t.fill_(-1)


@pytest.mark.parametrize("how", ["stream argument", "current stream"])
@pytest.mark.parametrize("case", CASES)
def test_launches_follow_the_work_of_their_stream(case, how):
    """The inputs arrive on the call's stream behind work that still runs when the call returns: a launch anywhere else
    meets NaN (and -1 as a length)."""
    inputs, outputs, scratch, call = CASES[case]()
    call(None)
    torch.cuda.synchronize()
    want, real = [t.clone() for t in outputs], [t.clone() for t in inputs]
    long = torch.ones((8192, 8192), device=DEV, dtype=BF16)
    torch.mm(long, long)
    s = torch.cuda.Stream()
    for products in (200, 1000, 4000):        # (more where the host was slow, or the call would prove nothing)
        for t in (*inputs, *outputs, *scratch):
            fill(t)
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


@pytest.mark.parametrize("case", CASES)
def test_the_marks_are_seen_and_implicit_streams(case):
    """On the inputs that a launch on another stream would meet every case gives other bytes; NULL, hipStreamLegacy and
    hipStreamPerThread give the same as a stream."""
    inputs, outputs, _, call = CASES[case]()
    real = [t.clone() for t in inputs]
    call(None)
    want = [t.clone() for t in outputs]
    for t in inputs:
        fill(t)
    call(None)
    torch.cuda.synchronize()
    assert any(not torch.equal(t.view(torch.uint8), w.view(torch.uint8)) for t, w in zip(outputs, want))
    for t, r in zip(inputs, real):
        t.copy_(r)
    for handle in (0, 1, 2):
        for t in outputs:
            fill(t)
        torch.cuda.synchronize()
        call(handle)
        torch.cuda.synchronize()
        assert all(torch.equal(t.view(torch.uint8), w.view(torch.uint8)) for t, w in zip(outputs, want)), handle


# -- offsets past 2^31 elements and 2^32 bytes ---------------------------------------------------------------------

ROWS, LD, LAST = 140000, 16392, 300      # 140000 * 16392 = 2.29e9 elements


def far(seed, std=1.0):
    """[ROWS, 64] of rows LD apart: random in the first and the last LAST rows, zeros between."""
    buf = torch.zeros((ROWS, LD), dtype=BF16, device=DEV)
    g = gen(seed)
    buf[0, :64] = normal(g, (64,), std)
    buf[-LAST:, :64] = normal(g, (LAST, 64), std)
    return buf[:, :64]


def far_empty():
    return torch.empty((ROWS, LD), dtype=BF16, device=DEV)[:, :64]


def test_far_offsets_norm_and_linear():
    x, y = far(1), far_empty()
    run_norm(x, None, None, None, 1e-6, y, 64)
    part = torch.cat((torch.arange(1), torch.arange(ROWS - LAST, ROWS))).to(DEV)
    _, want, err = R.layernorm(x[part], None, None, None, 1e-6)
    R.within(y[part], want, R.rounded(want, err, BF16), "y")
    dg, db, n = torch.empty(64, device=DEV), torch.empty(64, device=DEV), X.xema_layernorm_bwd_workspace_bytes(ROWS, 64)
    ws, dx = torch.empty(n, dtype=torch.uint8, device=DEV), far_empty()
    X.xema_op_layernorm_bwd(X.layernorm_bwd_args(x, 0, ROWS, 64, None, 1e-6, y, 0, dx, 0, dg, db, ws, n, ld_s=LD, ld_dy=LD, ld_dx=LD))
    want = R.layernorm_bwd(x[part], y[part], None, None, 1e-6)
    R.within(dx[part], want["dx"][0], R.rounded(*want["dx"], BF16), "dx")
    R.within(dg, *want["dgamma"], "dgamma")      # (the rows between add zeros)
    del dx
    w = normal(gen(3), (72, 64), 0.125)
    z = torch.empty((ROWS, LD), dtype=BF16, device=DEV)[:, :72]
    run_linear(x, w, None, 2, z)
    want = R.linear(x[part], w, None, 2, None)[2:]
    R.within(z[part], want[0], R.rounded(*want, BF16), "z")
    dw, dx = empty(72, 64, 0, BF16), y
    run_linear_bwd(x, w, None, z, 2, dx, dw, None)
    want = R.linear_bwd(x[part], w, None, z[part], 2, BF16)
    R.within(dx[part], want["dx"][0], R.rounded(*want["dx"], BF16), "dx")
    R.within(dw, want["dw"][0], R.rounded(*want["dw"], BF16), "dw")


@pytest.mark.parametrize("q_len", [3, 100])
def test_far_offsets_of_states(q_len):
    """Two sequences of 70000 states: the far rows hold the states that differ."""
    k, v = far(1), far(2)
    g = gen(5)
    q, do = normal(g, (2 * q_len, 64)), normal(g, (2 * q_len, 64))
    sizes, lens = (2, 1, 1, 64, q_len, ROWS // 2), torch.tensor([ROWS // 2, ROWS // 2 - 10], dtype=torch.int32, device=DEV)
    need = max(X.xema_cross_attn_workspace_bytes(*sizes), X.xema_cross_attn_bwd_workspace_bytes(*sizes))
    ws, o, lse = torch.empty(need, dtype=torch.uint8, device=DEV), empty(2 * q_len, 64, 0, BF16), torch.empty((2, 1, q_len), device=DEV)
    X.xema_op_cross_attn(X.cross_attn_args(0, *sizes, q, k, v, 0.125, o, ws, need, lse=lse, kv_lens=lens, ldk=LD, ldv=LD))
    ref = R.attention(q, k.contiguous(), v.contiguous(), 2, 1, 1, 64, lens, 0.125, BF16)
    R.within(o, ref["o"][0], R.rounded(*ref["o"], BF16), "o")
    dq, dk, dv = empty(2 * q_len, 64, 0, BF16), far_empty(), far_empty()
    X.xema_op_cross_attn_bwd(X.cross_attn_bwd_args(0, *sizes, q, k, v, 0.125, o, lse, do, dq, dk, dv, ws, need, kv_lens=lens, ldk=LD, ldv=LD,
                                                   ld_dk=LD, ld_dv=LD))
    ref = R.attention_bwd(q, k.contiguous(), v.contiguous(), o, lse, do, 2, 1, 1, 64, lens, 0.125, BF16)
    for n, t in (("dq", dq), ("dk", dk), ("dv", dv)):
        R.within(t, ref[n][0], R.rounded(*ref[n], BF16), n)


def test_far_offsets_of_tokens():
    q, do = far(1), far(2)
    g = gen(6)
    k, v = normal(g, (40, 64)), normal(g, (40, 64))
    sizes = (1, 1, 1, 64, ROWS, 40)
    need = max(X.xema_cross_attn_workspace_bytes(*sizes), X.xema_cross_attn_bwd_workspace_bytes(*sizes))
    ws, o, lse = torch.empty(need, dtype=torch.uint8, device=DEV), far_empty(), torch.empty((1, 1, ROWS), device=DEV)
    X.xema_op_cross_attn(X.cross_attn_args(0, *sizes, q, k, v, 0.125, o, ws, need, lse=lse, ldq=LD, ldo=LD))
    part = torch.cat((torch.arange(1), torch.arange(ROWS - LAST, ROWS))).to(DEV)
    lens = torch.tensor([40], device=DEV)
    ref = R.attention(q[part], k, v, 1, 1, 1, 64, lens, 0.125, BF16)
    R.within(o[part], ref["o"][0], R.rounded(*ref["o"], BF16), "o")
    dq, dk, dv = far_empty(), empty(40, 64, 0, BF16), empty(40, 64, 0, BF16)
    X.xema_op_cross_attn_bwd(X.cross_attn_bwd_args(0, *sizes, q, k, v, 0.125, o, lse, do, dq, dk, dv, ws, need, ldq=LD, ldo=LD, ld_do=LD, ld_dq=LD))
    ref = R.attention_bwd(q[part], k, v, o[part], lse[:, :, part], do[part], 1, 1, 1, 64, lens, 0.125, BF16)
    R.within(dq[part], ref["dq"][0], R.rounded(*ref["dq"], BF16), "dq")
    for n, t in (("dk", dk), ("dv", dv)):      # (the rows between have no dout: they add zeros)
        R.within(t, ref[n][0], R.rounded(*ref[n], BF16), n)
