"""The range and precision that xema_ffn.h states for t = scale x a^T, for few
rows and for many: fp16's largest, its finest, and bf16 at fp32's range."""
import pytest
import torch

import ffn_reference as R
from test_gpu_ffn import BF16, DEV, F16, empty, lora_inputs, run_lora, spread_ids

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 40, 300, 2600])
@pytest.mark.parametrize("dtype,scale", [(F16, 2.0 ** -12), (F16, 2.0 ** -20), (F16, 2.0 ** -26), (BF16, 2.0 ** -40), (BF16, 2.0 ** 40)])
def test_small_and_large_t(rows, dtype, scale):
    d = lora_inputs(rows, 264, 392, 16, 12, dtype, rows)
    d["scale"].fill_(scale)
    if scale > 1:       # (a y in range beside it)
        d["b"].mul_(1 / scale)
    else:               # the adapter's part alone: the projection adds nothing
        d["w"].zero_()
        d["bias"] = None
    ids = spread_ids(rows, 12, "mixed", rows)
    y = empty(rows, 392, 0, dtype)
    run_lora(d, ids, y)
    want, e = R.lora(d["x"], d["w"], d["bias"], d["a"], d["b"], d["scale"], ids, dtype)
    live = ids >= -1
    R.within(y[live], want[live], R.rounded(want, e, dtype)[live], "y")


@pytest.mark.parametrize("rows", [3, 300, 2600])
def test_the_largest_t_in_fp16(rows):
    """t of 65504, 65519 and -65519 whole, 65520 an infinity; an id each, the rest without."""
    d = lora_inputs(rows, 64, 392, 16, 4, F16, 1)
    for n in ("x", "w", "a", "b"):
        d[n] = torch.zeros_like(d[n])
    d["bias"] = None
    d["scale"].fill_(1)
    d["x"][:, 0], d["x"][:, 1] = 32752, 1
    d["a"][:, 3, 0] = torch.tensor([2, 2, -2, 2], device=DEV)
    d["a"][:, 3, 1] = torch.tensor([0, 15, -15, 16], device=DEV)
    d["b"][:, :, 3] = 2.0 ** -6
    t = torch.tensor([65504, 65519, -65519, float("inf")], device=DEV)
    ids = torch.arange(rows, device=DEV, dtype=torch.int32) % 5 - 1
    y = empty(rows, 392, 0, F16)
    run_lora(d, ids, y)
    want = torch.cat((torch.zeros(1, device=DEV), t * 2.0 ** -6))[(ids + 1).long()].to(F16)
    assert torch.equal(y, want[:, None].expand(-1, 392))
