"""The feed-forward products on the tiles, splits and few-row kernels that the
sizes of test_gpu_ffn.py do not reach (test_ffn_variants.py shows that both
together reach all of them), against the definitions in 64 bits."""
import pytest
import torch

import ffn_reference as R
from test_gpu_ffn import BF16, F16, F32, empty, gap_kept, gated_inputs, gen, lora_inputs, normal, pack24, run_bwd, run_lora, spread_ids, strided, unpack24

pytestmark = pytest.mark.gpu

# rows, dim, hidden: split products of the weights' gradients and of dx on every tile, and two layers of real sizes
BWD_SIZES = [(23466, 136, 1128), (9222, 136, 680), (20152, 72, 1104), (4231, 72, 968), (4316, 144, 5232), (65, 4160, 2200), (4196, 72, 4264),
             (32, 2072, 4080), (14125, 1008, 1744), (30000, 512, 1024)]


@pytest.mark.parametrize("rows,dim,hidden", BWD_SIZES)
@pytest.mark.parametrize("dtype,act", [(BF16, 1), (F16, 0)])
def test_gated_ffn_bwd(rows, dim, hidden, dtype, act):
    x, wg, wu, _, _ = gated_inputs(rows, dim, hidden, dtype, False, rows + dim)
    pre = pack24(normal(gen(rows), (rows, 2 * hidden), 1.5, F32))
    dy = strided(normal(gen(rows + 1), (rows, hidden), 0.5, dtype), 24)[0]
    out = run_bwd(x, wg, wu, pre, dy, act)
    want = R.gated_bwd(x, wg, wu, unpack24(pre, hidden), dy, act, dtype)
    for n in ("dgate_b", "dup_b", "dx", "dgate_w", "dup_w"):
        v, e = want[n]
        got = out[n][:, :dim] if n == "dx" else out[n]
        R.within(got, v, R.rounded(v, e, got.dtype), n)
    gap_kept(out["dx"], dim)
    again = run_bwd(x, wg, wu, pre, dy, act)
    assert all(torch.equal(again[n].view(torch.int16), out[n].view(torch.int16)) for n in want)


# rows, dim, out_dim, rank, adapters: reductions of every block, few rows of every block
LORA_SIZES = [(2000, 72, 136, 96, 4), (3000, 72, 136, 128, 4), (1400, 264, 72, 72, 5), (12400, 72, 72, 8, 3), (4200, 72, 72, 8, 3),
              (24, 1032, 392, 16, 3), (32, 136, 4096, 128, 5), (17, 72, 8200, 24, 3)]


@pytest.mark.parametrize("rows,dim,out_dim,rank,n", LORA_SIZES)
@pytest.mark.parametrize("how", ["one", "runs", "mixed"])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_lora_linear(rows, dim, out_dim, rank, n, how, dtype):
    d = lora_inputs(rows, dim, out_dim, rank, n, dtype, rows + dim, bias=rows % 2 == 0)
    ids = spread_ids(rows, n, how, rows)
    y = empty(rows, out_dim, 16, dtype)
    before = y.clone()
    run_lora(d, ids, y)
    want, e = R.lora(d["x"], d["w"], d["bias"], d["a"], d["b"], d["scale"], ids, dtype)
    live = ids >= -1
    R.within(y[live][:, :out_dim], want[live], R.rounded(want, e, dtype)[live], "y")
    assert torch.equal(y[~live].view(torch.int16), before[~live].view(torch.int16))
    gap_kept(y, out_dim)
