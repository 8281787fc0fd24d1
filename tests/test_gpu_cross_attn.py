"""Attention to an encoder's states and its gradient against their definitions in
64 bits: odd lengths and head dims, shared heads, ragged and empty sequences,
column ranges of one buffer, NaN behind the last state, single tokens."""
import math

import pytest
import torch

import cross_reference as R
import paper_2607_11136_amd as X
from test_gpu_ffn import BF16, CODE, DEV, F16, empty, gap_kept, gen, normal

pytestmark = pytest.mark.gpu


class Call:
    """One attention call's buffers: k and v column ranges of one buffer, gaps between all rows."""

    def __init__(self, batch, heads, kv_heads, d, q_len, kv_len, dtype, lens=None, seed=0, gap=8, spread=1.5):
        g = gen(seed + 31 * q_len + kv_len)
        self.sizes = (batch, heads, kv_heads, d, q_len, kv_len)
        self.dtype, self.scale = dtype, d ** -0.5
        nq, nk = heads * d, kv_heads * d
        self.nq, self.nk, self.gap = nq, nk, gap

        def rows(n, width, std):
            buf = torch.full((n, width + gap), 3.0, device=DEV).to(dtype)
            buf[:, :width] = normal(g, (n, width), std, dtype)
            return buf

        self.q = rows(batch * q_len, nq, spread)
        self.kv = rows(batch * kv_len, 2 * nk, 1.0)
        self.do = rows(batch * q_len, nq, 0.5)
        self.k, self.v = self.kv[:, :nk], self.kv[:, nk:2 * nk]
        self.lens = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
        self.o, self.lse = empty(batch * q_len, nq, gap, dtype), torch.full((batch, heads, q_len), 7.0, device=DEV)
        self.dq, self.dkv = empty(batch * q_len, nq, gap, dtype), empty(batch * kv_len, 2 * nk, gap, dtype)
        self.ws = torch.full((max(X.xema_cross_attn_workspace_bytes(*self.sizes), X.xema_cross_attn_bwd_workspace_bytes(*self.sizes), 256),), 0xFF,
                             dtype=torch.uint8, device=DEV)

    def true_lens(self):
        b, n = self.sizes[0], self.sizes[5]
        return torch.full((b,), n, device=DEV) if self.lens is None else self.lens.clamp(0, n)

    def forward(self, stream=None):
        lq, lk = self.nq + self.gap, 2 * self.nk + self.gap
        X.xema_op_cross_attn(X.cross_attn_args(CODE[self.dtype], *self.sizes, self.q, self.k, self.v, self.scale, self.o, self.ws, self.ws.numel(),
                                               lse=self.lse, kv_lens=self.lens, ldq=lq, ldk=lk, ldv=lk, ldo=lq), stream)

    def backward(self, stream=None, dq=True, dkv=True):
        lq, lk = self.nq + self.gap, 2 * self.nk + self.gap
        dk, dv = (self.dkv, self.dkv[:, self.nk:]) if dkv else (None, None)
        X.xema_op_cross_attn_bwd(X.cross_attn_bwd_args(CODE[self.dtype], *self.sizes, self.q, self.k, self.v, self.scale, self.o, self.lse, self.do,
                                                       self.dq if dq else None, dk, dv, self.ws, self.ws.numel(), kv_lens=self.lens, ldq=lq, ldk=lk,
                                                       ldv=lk, ldo=lq, ld_do=lq, ld_dq=lq, ld_dk=lk, ld_dv=lk), stream)

    def check_forward(self):
        b, h, kh, d, _, _ = self.sizes
        ref = R.attention(self.q[:, :self.nq], self.k, self.v, b, h, kh, d, self.true_lens(), self.scale, self.dtype)
        R.within(self.o[:, :self.nq], ref["o"][0], R.rounded(*ref["o"], self.dtype), "o")
        gap_kept(self.o, self.nq)
        want, bound = ref["lse"]
        none = torch.isinf(want)
        assert torch.equal(torch.isinf(self.lse) & (self.lse < 0), none)
        R.within(torch.where(none, 0.0, self.lse.double()), torch.where(none, 0.0, want), torch.where(none, 0.0, bound), "lse")

    def check_backward(self):
        b, h, kh, d, _, _ = self.sizes
        ref = R.attention_bwd(self.q[:, :self.nq], self.k, self.v, self.o[:, :self.nq], self.lse, self.do[:, :self.nq], b, h, kh, d, self.true_lens(),
                              self.scale, self.dtype)
        for name, got in (("dq", self.dq[:, :self.nq]), ("dk", self.dkv[:, :self.nk]), ("dv", self.dkv[:, self.nk:2 * self.nk])):
            R.within(got, ref[name][0], R.rounded(*ref[name], self.dtype), name)
        gap_kept(self.dq, self.nq)
        gap_kept(self.dkv, 2 * self.nk)


# batch, heads, kv_heads, head_dim, q_len, kv_len, lens
SIZES = [
    (1, 1, 1, 8, 1, 1, None), (1, 1, 1, 64, 1, 63, None), (1, 2, 1, 128, 3, 65, None), (2, 4, 4, 64, 33, 1, [1, 0]),
    (2, 3, 3, 72, 65, 77, [77, 30]), (3, 4, 2, 40, 130, 129, [129, 64, 0]), (2, 6, 2, 96, 257, 200, [1, 199]), (1, 2, 2, 104, 300, 64, None),
    (2, 2, 1, 128, 500, 300, [300, 128]), (1, 3, 3, 24, 129, 1000, None), (2, 8, 1, 128, 70, 515, [400, 515]), (4, 2, 2, 64, 1030, 31, [31, 5, 0, 32]),
    (1, 16, 4, 56, 16, 700, [-3]), (1, 2, 2, 120, 600, 1100, [2000]), (8, 40, 40, 64, 90, 40, None),
    (1, 2, 2, 64, 300, 900, None), (1, 2, 2, 88, 200, 1000, None), (1, 2, 1, 32, 700, 100, None),
    (1, 2, 2, 64, 300, 1025, [1000]), (1, 2, 2, 88, 200, 1300, None), (1, 3, 3, 32, 129, 1200, [1100]), (1, 2, 2, 120, 200, 2100, None),
    (8, 33, 33, 32, 40, 20, None), (4, 99, 33, 32, 70, 20, [20, 3, 0, 9]), (4, 99, 33, 56, 70, 20, [7, 20, 20, 1]), (8, 33, 33, 72, 40, 20, None),
    (4, 99, 33, 96, 70, 20, [0, 20, 11, 20]),
]
TOKENS = [
    (1, 1, 1, 128, 1, 1, None), (3, 8, 1, 128, 1, 5000, [5000, 1, 0]), (2, 4, 4, 64, 1, 3001, [3001, 64]), (1, 32, 8, 128, 1, 9000, None),
    (2, 6, 3, 72, 5, 1027, [1000, 33]), (4, 16, 2, 96, 4, 513, [0, 512, 513, 31]), (2, 64, 1, 32, 1, 2000, [2000, 1999]), (130, 4, 2, 64, 1, 40, None),
    (2, 8, 2, 88, 3, 250, [250, 7]), (2, 8, 2, 96, 3, 100, [100, 7]),
]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("size", SIZES + TOKENS, ids=str)
def test_forward(size, dtype):
    c = Call(*size[:6], dtype, size[6])
    c.forward()
    c.check_forward()


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("size", SIZES + TOKENS[1:6], ids=str)
def test_gradient(size, dtype):
    c = Call(*size[:6], dtype, size[6], seed=1)
    c.forward()
    c.backward()
    c.check_backward()


def test_gradient_against_differences():
    """The formula's own gradient in 64 bits meets central differences of the loss sum(do * o)."""
    c = Call(2, 4, 2, 16, 5, 9, F16, [9, 4])
    b, h, kh, d, _, _ = c.sizes
    lens = c.true_lens()
    q, k, v, do = (t.double().clone() for t in (c.q[:, :c.nq], c.k, c.v, c.do[:, :c.nq]))

    def forward():
        return R.attention(q, k, v, b, h, kh, d, lens, c.scale, F16)

    o, lse = forward()["o"][0], forward()["lse"][0]
    want = R.attention_bwd(q, k, v, o, lse, do, b, h, kh, d, lens, c.scale, F16)
    for name, t in (("dq", q), ("dk", k), ("dv", v)):
        for i, j in ((0, 0), (3, 17), (t.shape[0] - 1, t.shape[1] - 1), (4, 5)):
            x = float(t[i, j])
            loss = []
            for s in (1e-4, -1e-4):
                t[i, j] = x + s
                loss.append(float((do * forward()["o"][0]).sum()))
            t[i, j] = x
            # a third derivative of order 1 leaves 1e-8 of it
            assert abs((loss[0] - loss[1]) / 2e-4 - float(want[name][0][i, j])) < 1e-6, (name, i, j)


@pytest.mark.parametrize("size", [(1, 2, 2, 64, 40, 200, None), (2, 8, 2, 128, 1, 700, [700, 300]), (1, 2, 1, 128, 300, 130, None)], ids=str)
def test_one_state_takes_all(size):
    """A query that meets one state far above the others gives that state's v, and the state its gradient."""
    c = Call(*size[:6], F16, size[6], spread=0.0)
    b, h, kh, d, q_len, kv_len = c.sizes
    lens = c.true_lens().tolist()
    c.q[:, :c.nq] = 0
    c.k[:] = 0
    chosen = {}
    for i in range(b):
        for t in range(q_len):
            for x in range(h):
                # state j has 100 at one place and its index's bits as signs; the query is a multiple of it
                chosen[i, t, x] = (7 * t + 11 * x + 3) % lens[i]
    for i in range(b):
        for j in range(lens[i]):
            bits = torch.tensor([1.0 if j >> s & 1 else -1.0 for s in range(d)], device=DEV)
            for g in range(kh):
                c.k[i * kv_len + j, g * d:(g + 1) * d] = 4 * bits
    for (i, t, x), j in chosen.items():
        c.q[i * q_len + t, x * d:(x + 1) * d] = c.k[i * kv_len + j, (x // (h // kh)) * d:(x // (h // kh) + 1) * d] * 16
    c.forward()
    # two indexes differ in one bit at least: scores differ by 2 * 4 * 64 / sqrt(d) > 45, a weight under 2^-64
    o = c.o[:, :c.nq].float()
    dv, mag = (torch.zeros((b * kv_len, c.nk), dtype=torch.float64, device=DEV) for _ in range(2))
    for (i, t, x), j in chosen.items():
        at = (x // (h // kh)) * d
        assert torch.equal(o[i * q_len + t, x * d:(x + 1) * d], c.v[i * kv_len + j, at:at + d].float()), (i, t, x, j)
        do = c.do[i * q_len + t, x * d:(x + 1) * d].double()
        dv[i * kv_len + j, at:at + d] += do
        mag[i * kv_len + j, at:at + d] += do.abs()
    c.backward()
    got = c.dkv[:, c.nk:2 * c.nk].double()
    # every product is a whole number, so s is exact; scale * s reaches 4 * 64 * sqrt(d) < 2900: s, lse and their
    # difference in fp32 leave p = 1 off by 16 U of that, and its rounding to the type by half a step
    bound = (16 * R.U * 2900 + R.HALF[F16] + 700 * 2 * R.U) * mag
    R.within(got, dv, R.rounded(dv, bound, F16), "dv")


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("size", [(2, 3, 3, 72, 65, 150, [100, 0]), (2, 4, 2, 128, 1, 900, [130, 33]), (1, 2, 2, 64, 300, 70, [1])], ids=str)
def test_nan_behind_the_last_state(size, dtype):
    c = Call(*size[:6], dtype, size[6], seed=2)
    for bad in (float("nan"), float("inf"), float("-inf"), torch.finfo(dtype).min):
        for i, n in enumerate(size[6]):
            c.kv[i * size[5] + n:(i + 1) * size[5], :2 * c.nk] = bad
        c.forward()
        c.check_forward()
        c.backward()
        c.check_backward()


def test_non_finite_values_where_they_are_met():
    c = Call(1, 2, 2, 64, 130, 90, BF16, None, seed=3)
    c.q[5, 3] = float("nan")           # a query of head 0
    c.v[7, 64 + 2] = float("inf")      # a state's value in head 1, column 2
    c.forward()
    o = c.o[:, :c.nq].float()
    assert bool(torch.isnan(o[5, :64]).all()) and bool(torch.isfinite(o[4, :64]).all()) and bool(torch.isfinite(o[6:, :64]).all())
    head = o[:, 64:]
    assert bool((head[:, 2] == float("inf")).all())
    head = torch.cat((head[:, :2], head[:, 3:]), 1)
    assert bool(torch.isfinite(head).all())


def test_scores_of_minus_infinity():
    """They weigh nothing; a token of nothing else gives zeros and no NaN."""
    c = Call(1, 1, 1, 64, 40, 100, BF16, None, seed=4, gap=0)
    c.q[:] = 1.0
    c.k[:, :] = 0.25
    c.k[10:30] = float("-inf")
    c.forward()
    want = torch.cat((c.v[:10], c.v[30:])).double().mean(0).expand(40, 64)
    mag = torch.cat((c.v[:10], c.v[30:])).double().abs().mean(0).expand(40, 64)
    R.within(c.o, want, R.rounded(want, mag * (R.HALF[BF16] + 200 * R.U), BF16), "o")
    c.k[:] = float("-inf")
    c.forward()
    assert bool((c.o == 0).all()) and bool((c.lse == float("-inf")).all())
    c.backward()
    assert bool((c.dkv == 0).all())


@pytest.mark.parametrize("size", [(2, 4, 2, 64, 100, 90, [90, 40]), (1, 8, 8, 128, 20, 4000, None), (1, 2, 2, 72, 3000, 20, None)], ids=str)
def test_parts_of_the_gradient(size):
    """dq alone, and dk and dv alone, have the bytes that they have together."""
    c = Call(*size[:6], BF16, size[6], seed=5)
    c.forward()
    c.backward()
    want = [c.dq.clone(), c.dkv.clone()]
    for dq, dkv in ((True, False), (False, True)):
        c.dq.view(torch.uint8).fill_(0xFF)
        c.dkv.view(torch.uint8).fill_(0xFF)
        c.ws.fill_(0xAA)
        c.backward(dq=dq, dkv=dkv)
        for t, w, there in ((c.dq, want[0], dq), (c.dkv, want[1], dkv)):
            assert torch.equal(t.view(torch.uint8), w.view(torch.uint8)) if there else bool((t.view(torch.uint8) == 0xFF).all())


def test_no_states_and_no_tokens():
    c = Call(2, 4, 2, 64, 33, 8, BF16)
    b, h, kh, d, q_len, _ = c.sizes
    lq = c.nq + c.gap
    X.xema_op_cross_attn(X.cross_attn_args(0, b, h, kh, d, q_len, 0, c.q, c.k, c.v, 0.1, c.o, lse=c.lse, ldq=lq, ldo=lq))
    assert bool((c.o[:, :c.nq] == 0).all()) and bool((c.lse == float("-inf")).all())
    lk = 2 * c.nk + c.gap
    X.xema_op_cross_attn_bwd(X.cross_attn_bwd_args(0, b, h, kh, d, 0, 8, c.q, c.k, c.v, 0.1, c.o, c.lse, c.do, c.dq, c.dkv, c.dkv[:, c.nk:], c.ws,
                                                   c.ws.numel(), ldk=lk, ldv=lk, ld_dk=lk, ld_dv=lk))
    assert bool((c.dkv[:, :2 * c.nk] == 0).all())
    gap_kept(c.dkv, 2 * c.nk)
    c.dq.view(torch.uint8).fill_(0xFF)
    X.xema_op_cross_attn_bwd(X.cross_attn_bwd_args(0, b, h, kh, d, q_len, 0, c.q, c.k, c.v, 0.1, c.o, c.lse, c.do, c.dq, c.dkv, c.dkv[:, c.nk:], c.ws,
                                                   c.ws.numel(), ldq=lq, ldo=lq, ld_do=lq, ld_dq=lq))
    assert bool((c.dq[:, :c.nq] == 0).all())
    gap_kept(c.dq, c.nq)


def test_large_scores_and_moving_maxima():
    """States in rising order of their score, by hundreds: every tile moves the reference."""
    for dtype in (BF16, F16):
        c = Call(1, 2, 2, 64, 200, 640, dtype, None, seed=6, gap=0)
        ramp = torch.arange(640, device=DEV).float()[:, None] / 640
        for order in (ramp, 1 - ramp):
            c.k[:, 0] = (order[:, 0] * 60).to(dtype)
            c.k[:, 64] = (order[:, 0] * 60).to(dtype)
            c.q[:, 0], c.q[:, 64] = 60.0, -60.0
            c.forward()
            c.check_forward()
            c.backward()
            c.check_backward()
    assert math.isfinite(float(c.lse.abs().max()))


def test_small_probabilities_keep_their_bits_in_fp16():
    """20000 states of like weight: p = 5e-5 is below fp16's normal range, 2^14 p is not."""
    c = Call(1, 1, 1, 64, 64, 20000, F16, None, seed=7, gap=0, spread=0.05)
    c.do.mul_(8)
    c.forward()
    c.check_forward()
    c.backward()
    p = 1 / 20000
    want = R.attention_bwd(c.q, c.k, c.v, c.o, c.lse, c.do, 1, 1, 1, 64, c.true_lens(), c.scale, F16)["dv"][0]
    # 64 terms of p do: each off by 2^-11 of it at most; the rounding of dv, whose own values lie near fp16's smallest
    bound = 64 * p * c.do.double().abs().amax() * (2 * R.HALF[F16]) + R.HALF[F16] * want.abs() + R.TINY[F16]
    R.within(c.dkv[:, 64:], want, bound.expand_as(want), "dv")
