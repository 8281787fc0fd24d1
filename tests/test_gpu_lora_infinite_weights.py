"""Adapters whose b holds infinities and NaN: which outputs are infinite, of
which sign, and which are NaN is the formula's answer on every path, for few
rows and for many, for a wave's first three adapters and for further ones."""
import pytest
import torch

import ffn_reference as R
from test_gpu_ffn import BF16, DEV, F16, empty, lora_inputs, run_lora, spread_ids

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")
# (column, its ranks with other values): one infinity, one of the other sign, two alike, two unlike, a NaN alone and beside one
SPECIAL = [(3, {0: INF}), (9, {5: -INF}), (17, {1: INF, 6: INF}), (40, {2: INF, 7: -INF}), (64, {4: NAN}), (71, {0: INF, 3: NAN})]

# few rows of both widths and the first sizes past them, sizes that reach every tile, and a last rank step of 8 of 32
SIZES = [(1, 264, 392, 16), (16, 72, 8264, 8), (48, 264, 392, 8), (64, 136, 4104, 16), (33, 64, 8264, 16), (65, 264, 392, 16), (130, 328, 520, 64),
         (300, 264, 392, 24), (582, 72, 3376, 8), (700, 256, 2056, 128), (1500, 192, 4104, 40), (9000, 256, 1544, 16), (12500, 136, 520, 32)]


@pytest.mark.parametrize("rows,dim,out_dim,rank", SIZES)
@pytest.mark.parametrize("how", ["one", "runs", "mixed"])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_infinite_weights(rows, dim, out_dim, rank, how, dtype):
    n = 12 if how == "mixed" else 3
    d = lora_inputs(rows, dim, out_dim, rank, n, dtype, rows + rank)
    ids = spread_ids(rows, n, how, rows)
    ids[0] = n - 1                              # (a single row too has an adapter)
    marked = [n - 1] if n == 3 else range(0, n, 2)
    finite = {**d, "b": d["b"].clone()}
    for i in marked:
        for c, ranks in SPECIAL:
            for q, v in ranks.items():
                d["b"][i, c, q], finite["b"][i, c, q] = v, 0
    y = empty(rows, out_dim, 0, dtype)
    run_lora(d, ids, y)

    want, e = R.lora(finite["x"], finite["w"], finite["bias"], finite["a"], finite["b"], finite["scale"], ids, dtype)
    live = ids >= -1
    plain = torch.ones(out_dim, dtype=torch.bool, device=DEV)
    plain[[c for c, _ in SPECIAL]] = False
    R.within(y[live][:, plain], want[live][:, plain], R.rounded(want, e, dtype)[live][:, plain], "columns of finite weights")
    for i in range(n):
        mine = (ids == i).nonzero()[:, 0]
        if not len(mine):
            continue
        # t's sign decides: rows in which a t beside an infinity is within its error of 0 are left out
        t, et = R.product(d["x"][mine], d["a"][i], 2)
        sure = t.abs() > et + R.TINY[dtype] * 4
        for c, ranks in SPECIAL:
            got = y[mine, c].double()
            if i not in marked:
                assert bool(torch.isfinite(got).all())
                continue
            special = sum(t[:, q] * v for q, v in ranks.items())        # (inf - inf is NaN here as there)
            use = sure[:, list(ranks)].all(1)
            assert float(use.double().mean()) > 0.9 or len(mine) < 30
            assert torch.equal(torch.isnan(got[use]), torch.isnan(special[use])), (i, c)
            assert torch.equal(torch.nan_to_num(got[use], 0.0, 1.0, -1.0), torch.nan_to_num(special[use], 0.0, 1.0, -1.0)), (i, c)


@pytest.mark.parametrize("rows", [40, 300, 2600])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_infinite_rows_meet_infinite_weights(rows, dtype):
    """x a^T infinite beside an infinite b: an infinity of the signs' product."""
    d = lora_inputs(rows, 264, 392, 16, 2, dtype, rows)
    for k in ("x", "w", "a", "b"):
        d[k] = d[k].abs() + 2.0 ** -10
    d["x"][1, 5] = INF
    d["b"][:, 7, 3], d["b"][:, 8, 4] = INF, -INF
    ids = spread_ids(rows, 2, "mixed", rows)
    ids[1] = 0
    y = empty(rows, 392, 0, dtype)
    run_lora(d, ids, y)
    want = torch.full((392,), INF, device=DEV, dtype=dtype)
    want[8] = NAN                               # (the other ranks' infinities, and this one's)
    assert torch.equal(torch.isnan(y[1]), torch.isnan(want)) and bool((y[1][torch.arange(392, device=DEV) != 8] == INF).all())
    named = ids >= 0
    named[1] = False
    assert bool((y[named][:, 7] == INF).all()) and bool((y[named][:, 8] == -INF).all())
