"""The RMS norm and its gradient with every type of every argument, at each number of vectors and waves that a row takes:
the kernels store by a type that they learn at run time, between sums that they go on with."""
import pytest
import torch

import ffn_reference as R
import paper_2607_11136_amd as X
from test_gpu_ffn import BF16, CODE, DEV, F16, F32, empty, gen, normal, run_norm

pytestmark = pytest.mark.gpu

TYPES = (BF16, F16, F32)


@pytest.mark.parametrize("dim", [264, 520, 1032, 2056, 4104, 8200])
def test_every_type_at_every_width(dim):
    rows, g = 19, gen(dim)
    gamma = normal(g, (dim,), 0.3, mean=1.0)
    s, dy, dsum = ({t: normal(g, (rows, dim), std, t, mean) for t in TYPES} for std, mean in ((2.0, -0.7), (0.5, 0.1), (0.3, 0.0)))
    n = X.xema_rmsnorm_bwd_workspace_bytes(rows, dim)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    for st in TYPES:
        for dt in TYPES:
            for at in (None, *TYPES):
                want = R.rmsnorm_bwd(s[st], dy[dt], dsum[at] if at else None, gamma, 1e-5)
                for ot in TYPES:
                    dx, dgamma = empty(rows, dim, 0, ot), torch.full((dim,), 7.0, device=DEV)
                    X.xema_op_rmsnorm_bwd(X.rmsnorm_bwd_args(s[st], CODE[st], rows, dim, gamma, 1e-5, dy[dt], CODE[dt], dx, CODE[ot], dgamma, ws, n,
                                                             dsum=dsum[at] if at else None, dsum_dtype=CODE[at] if at else 0))
                    R.within(dx, want["dx"][0], R.rounded(*want["dx"], ot), ("dx", st, dt, at, ot))
                    R.within(dgamma, *want["dgamma"], ("dgamma", st, dt, at, ot))
            for yt in (BF16, F16):
                for sumt in (None, *TYPES):
                    for resid in (None, dy[dt]):
                        y, total = empty(rows, dim, 0, yt), empty(rows, dim, 0, sumt) if sumt else None
                        run_norm(s[st], resid, gamma, 1e-5, y, dim, total)
                        want_s, want, rel = R.rmsnorm(s[st], resid, gamma, 1e-5)
                        R.within(y, want, R.rounded(want, rel * want.abs(), yt), ("y", st, dt, yt, sumt))
                        if sumt:
                            R.within(total, want_s, R.rounded(want_s, R.U * want_s.abs(), sumt), ("sum", st, dt, sumt))
