"""Attention whose parts are joined many rows at a time, behind the kernel of single tokens and behind that of blocks of
queries: ragged sequences, some of which leave parts empty, and workspaces that hold NaN before the call."""
import pytest
import torch

from test_gpu_cross_attn import Call
from test_gpu_ffn import BF16, F16

pytestmark = pytest.mark.gpu

# batch, heads, kv_heads, head_dim, q_len, kv_len, lens: more than 1024 (batch, head, token) rows (tests/test_cross_joins.py)
SIZES = [
    (5, 21, 21, 64, 15, 5625, [5625, 1, 0, 700, 5624]), (9, 32, 8, 40, 4, 600, [600, 599, 1, 0, 33, 128, 129, 500, 31]),
    (4, 12, 12, 96, 24, 2000, [2000, 3, 0, 777]), (9, 32, 8, 128, 4, 600, [33, 600, 0, 1, 64, 255, 256, 257, 600]),
    (1, 4, 2, 64, 300, 1100, [900]), (2, 2, 1, 40, 400, 2000, [2000, 33]), (2, 3, 3, 88, 200, 1500, [1500, 0]), (1, 4, 4, 128, 300, 1030, None),
]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_joined_rows(size, dtype):
    c = Call(*size[:6], dtype, size[6], seed=21)
    c.forward()
    c.check_forward()
    o, lse = c.o[:, :c.nq].clone(), c.lse.clone()
    c.o.view(torch.uint8).fill_(0xFF)
    c.ws.fill_(0xAA)
    c.forward()
    assert torch.equal(c.o[:, :c.nq].view(torch.int16), o.view(torch.int16)) and torch.equal(c.lse.view(torch.int32), lse.view(torch.int32))
