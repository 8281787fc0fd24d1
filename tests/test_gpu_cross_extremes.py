"""Attention to an encoder's states where its scores are extreme: finite ones as far
as fp32 goes, of either sign, in every kernel of the forward pass."""
import pytest
import torch

import cross_reference as R
from test_gpu_cross_attn import Call
from test_gpu_ffn import BF16, DEV, F16, gen

pytestmark = pytest.mark.gpu

# blocks of queries and single tokens, whole and in parts, the parts joined row by row and many rows at a time
KERNELS = [(2, 4, 2, 64, 130, 200, [200, 77]), (1, 2, 2, 96, 100, 2100, [2050]), (1, 3, 3, 64, 500, 1100, None), (1, 2, 2, 128, 600, 1100, None),
           (3, 4, 2, 64, 1, 100, [100, 1, 33]), (1, 4, 2, 128, 2, 3000, [2500])]


def levels(c, base, seed):
    """Scores of base * scale times 1, 1.25, 1.5 or 1.75 by the state, exact in fp32; the states whose score is the highest, by
    sequence."""
    b, _, kh, d, _, n = c.sizes
    times = 1 + 0.25 * torch.randint(0, 4, (b * n,), generator=gen(seed), device=DEV)
    c.q[:, :c.nq] = 0
    c.k[:] = 0
    root = 1.0 if c.dtype == BF16 else 2.0 ** 15         # (fp16: both factors share the score)
    c.q[:, 0:c.nq:d] = root
    c.k[:, 0:c.nk:d] = (times * (base / root)).to(c.dtype)[:, None]
    s = c.k[:, 0].double() * root
    top = []
    for i, m in enumerate(c.true_lens().tolist()):
        mine = s[i * n:i * n + m]
        top.append((mine == mine.max(), float(mine.max()) * c.scale))
    return top


@pytest.mark.parametrize("size", KERNELS, ids=str)
@pytest.mark.parametrize("dtype,base", [(t, s * b) for s in (1, -1) for t, b in ((BF16, 1e7), (BF16, 2e8), (BF16, 1e10), (BF16, 1e20), (BF16, 1e30),
                                                                                 (BF16, 1e38), (F16, 1e7), (F16, 1e9))], ids=str)
def test_finite_scores_of_any_size(size, dtype, base):
    """The states of the highest score share the weight, and the others have none."""
    c = Call(*size[:6], dtype, size[6], seed=11)
    b, h, kh, d, q_len, n = c.sizes
    tops = levels(c, base, 5)
    c.forward()
    for i, (top, s) in enumerate(tops):
        v = c.v[i * n:i * n + top.numel()].double()[top].reshape(-1, kh, 1, d).expand(-1, kh, h // kh, d).reshape(-1, h * d)
        # the weights are one value, rounded once to the type; the sums of their products and their own are fp32
        want, mag = v.mean(0), v.abs().mean(0)
        bound = R.rounded(want, (R.HALF[dtype] + (n + 100) * 4 * R.U) * mag, dtype)
        o = c.o[i * q_len:(i + 1) * q_len, :c.nq]
        R.within(o, want.expand_as(o), bound.expand_as(o), "o")
        # the scale, times log2(e), times the score, the sum with the weights' part and the way back: six roundings
        lse = c.lse[i].double()
        want = s + torch.full_like(lse, len(v)).log()
        R.within(lse, want, 6 * R.U * want.abs() + (n + 100) * 2 * R.U, "lse")


# the kernels of the gradient: one launch and two, dq whole and in parts, dk and dv too, every width of heads
GRADIENTS = [(2, 4, 2, 64, 130, 200, [200, 77]), (1, 2, 2, 96, 100, 2100, [2050]), (8, 33, 33, 32, 40, 20, None), (8, 33, 33, 72, 40, 20, None),
             (1, 2, 2, 128, 3000, 20, None), (1, 16, 1, 128, 1100, 150, None), (1, 4, 2, 128, 2, 3000, [2500]), (4, 32, 32, 128, 300, 100, [100, 9, 50, 0])]


@pytest.mark.parametrize("size", GRADIENTS, ids=str)
@pytest.mark.parametrize("dtype,base", [(t, s * b) for s in (1, -1) for t, b in ((BF16, 1e8), (BF16, 1e10), (BF16, 1e30), (BF16, 1e36), (F16, 1e8),
                                                                                 (F16, 1e9))], ids=str)
def test_tokens_whose_lse_tells_no_weights_have_no_gradient(size, dtype, base):
    """Every third token has scores of +-base, with an lse past 2^22: the gradients are those of the other tokens alone."""
    c = Call(*size[:6], dtype, size[6], seed=12)
    b, h, kh, d, q_len, n = c.sizes
    root = 1.0 if dtype == BF16 else 2.0 ** 15           # (fp16: both factors share the score)
    c.k[:, 0:c.nk:d] = base / root
    c.q[:, 0:c.nq:d] = 0
    coarse = torch.arange(b * q_len, device=DEV) % 3 == 1
    c.q[coarse, 0:c.nq:d] = root
    c.forward()
    lse = c.lse.transpose(1, 2).reshape(b * q_len, h).abs()
    # (infinite where a sequence has no states)
    assert bool((lse[coarse] > 2.0 ** 22).all()) and bool(((lse < 100) | torch.isinf(lse))[~coarse].all())
    c.backward()
    assert bool((c.dq[coarse, :c.nq] == 0).all())
    # (the reference meets the other tokens alone: no dout, and scores and an lse that leave p = 0 here)
    c.q[coarse, :c.nq] = 0
    c.do[coarse] = 0
    c.lse[:] = torch.where(coarse.view(b, 1, q_len).expand(b, h, q_len), 1e4, c.lse)
    c.check_backward()


@pytest.mark.parametrize("size", GRADIENTS, ids=str)
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_gradient_of_scores_of_tens_of_thousands(size, dtype):
    """p comes from lse: the bound takes 4 half steps of it."""
    c = Call(*size[:6], dtype, size[6], seed=13)
    d = c.sizes[3]
    c.k[:, 0:c.nk:d] = 1000
    c.q[:, 0:c.nq:d] = torch.linspace(-500, 500, c.q.shape[0], device=DEV).to(dtype)[:, None]
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()
    assert float(c.lse.abs().max()) > 4e4


# with the states of the first part, where there are parts
@pytest.mark.parametrize("size,first", list(zip(KERNELS, (64, 288, 288, 288, 1, 128))), ids=str)
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_nan_of_any_state_is_met(size, first, dtype):
    """Every sequence's first states, a whole part of them, have NaN as keys, or as the values of states that weigh nothing in
    fp32: it is not lost where the parts are joined."""
    c = Call(*size[:6], dtype, size[6], seed=14)
    b, h, kh, d, q_len, n = c.sizes
    bad = (torch.arange(n, device=DEV) < first).repeat(b)
    keep = c.kv.clone()
    c.kv[bad, :c.nk] = float("nan")
    c.forward()
    assert bool(torch.isnan(c.o[:, :c.nq]).all()) and bool(torch.isnan(c.lse).all())
    c.kv.copy_(keep)
    c.q[:, 0:c.nq:d] = 100
    c.k[bad, 0:c.nk:d] = -100           # a weight of e^-883 at most beside the others
    c.v[bad, 1:c.nk:d] = float("nan")
    c.forward()
    o = c.o[:, :c.nq].view(-1, h, d)
    assert bool(torch.isnan(o[:, :, 1]).all()) and bool(torch.isfinite(torch.cat((o[:, :, :1], o[:, :, 2:]), 2)).all())
    assert bool(torch.isfinite(c.lse).all())
