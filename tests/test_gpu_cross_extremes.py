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
