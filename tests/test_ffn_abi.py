"""The feed-forward sub-block's entry points without a GPU: exports, the
documented refusals (all before any device work), workspace sizes."""
import ctypes
import os
import re

import pytest

import paper_2607_11136_amd as X

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MB = 1 << 20
INVALID, UNSUPPORTED, SMALL, MISALIGNED = (X.XEMA_ERR_INVALID_ARG, X.XEMA_ERR_UNSUPPORTED, X.XEMA_ERR_WORKSPACE_TOO_SMALL,
                                           X.XEMA_ERR_MISALIGNED)


def test_exports_are_those_of_the_header():
    src = open(os.path.join(ROOT, "include", "xema_ffn.h")).read()
    names = set(re.findall(r"XEMA_API\s+[\w\s\*]+?\b(xema_\w+)\s*\(", src))
    assert names == set(X.EXPORTED_FFN) and not names & set(X.EXPORTED)
    for n in names:
        assert hasattr(X.lib(), n), n


def test_structs_have_the_headers_fields():
    src = open(os.path.join(ROOT, "include", "xema_ffn.h")).read()
    for name, cls in (("xema_rmsnorm_args", X.RmsnormArgs), ("xema_rmsnorm_bwd_args", X.RmsnormBwdArgs),
                      ("xema_gated_ffn_args", X.GatedFfnArgs), ("xema_gated_ffn_bwd_args", X.GatedFfnBwdArgs),
                      ("xema_lora_args", X.LoraArgs)):
        body = re.search(r"typedef struct \{([^}]*)\} " + name + ";", src).group(1)
        fields = []
        for part in body.split(";"):
            m = re.match(r"\s*(const )?(int64_t|int32_t|float|void)\b(.*)", part, re.S)
            if m:
                fields += [(m.group(2) if "*" not in f else "*", f.strip(" *\n")) for f in m.group(3).split(",")]
        kinds = {"int64_t": ctypes.c_int64, "int32_t": ctypes.c_int32, "float": ctypes.c_float, "*": ctypes.c_void_p}
        pointer = re.findall(r"\*\s*(\w+)", body)
        assert [(n, ctypes.c_void_p if n in pointer else kinds[k]) for k, n in fields] == cls._fields_, name


# Addresses that nothing dereferences: every call here is refused, or has no rows.
def at(i):
    return (i + 1) << 32


def norm(**kw):
    a = dict(rows=0, dim=64, x=at(0), x_dtype=0, ldx=64, resid=at(1), resid_dtype=2, ld_resid=64, sum=at(2), sum_dtype=2, ld_sum=64,
             gamma=at(3), eps=1e-6, y=at(4), y_dtype=0, ldy=64, y_scale=None)
    a.update(kw)
    return "xema_op_rmsnorm", X.RmsnormArgs(**a)


def norm_bwd(**kw):
    a = dict(rows=0, dim=64, s=at(0), s_dtype=0, ld_s=64, dy=at(1), dy_dtype=0, ld_dy=64, dsum=at(2), dsum_dtype=0, ld_dsum=64, gamma=at(3),
             eps=1e-6, dx=at(4), dx_dtype=0, ld_dx=64, dgamma=None, workspace=None, workspace_bytes=0)
    a.update(kw)
    return "xema_op_rmsnorm_bwd", X.RmsnormBwdArgs(**a)


def gated(**kw):
    a = dict(dtype=0, act=0, rows=0, dim=64, hidden=128, x=at(0), ldx=64, x_scale=None, gate_w=at(1), up_w=at(2), gate_scale=None,
             up_scale=None, gate_b=at(3), up_b=at(4), y=at(5), y_dtype=0, ldy=128, pre=at(6))
    a.update(kw)
    return "xema_op_gated_ffn", X.GatedFfnArgs(**a)


def gated8(**kw):
    return gated(**{**dict(dtype=3, pre=None, x_scale=at(7), gate_scale=at(8), up_scale=at(9)), **kw})


def gated_bwd(**kw):
    a = dict(dtype=0, act=0, rows=0, dim=64, hidden=128, x=at(0), ldx=64, gate_w=at(1), up_w=at(2), pre=at(3), dy=at(4), ld_dy=128, dx=at(5),
             ld_dx=64, dgate_w=None, dup_w=None, dgate_b=None, dup_b=None, workspace=at(10), workspace_bytes=1 << 31)
    a.update(kw)
    return "xema_op_gated_ffn_bwd", X.GatedFfnBwdArgs(**a)


def lora(**kw):
    a = dict(dtype=0, rows=0, dim=64, out_dim=128, x=at(0), ldx=64, w=at(1), bias=at(2), a=at(3), b=at(4), scale=at(5), rank=16, n_adapters=3,
             row_adapter=at(6), y=at(7), y_dtype=0, ldy=128, workspace=at(8), workspace_bytes=1 << 31)
    a.update(kw)
    return "xema_op_lora_linear", X.LoraArgs(**a)


def call(case):
    name, args = case
    return getattr(X.lib(), name)(ctypes.byref(args), None)


@pytest.mark.parametrize("case", [norm(), norm(resid=None, sum=None, gamma=None), norm(y_dtype=3, y_scale=at(9)), norm_bwd(),
                                  norm_bwd(dsum=None, gamma=None), gated(), gated(gate_b=None, up_b=None, pre=None), gated8(),
                                  gated8(y_dtype=1), gated_bwd(), lora(), lora(n_adapters=0, a=None, b=None, scale=None, bias=None),
                                  lora(y_dtype=1), norm(rows=0, sum=at(1)), gated(up_w=at(1) + 64 * 128 * 2)])
def test_accepted_with_no_rows(case):
    assert call(case) == X.XEMA_OK


REFUSED = [
    (norm(rows=-1), INVALID), (norm(rows=1 << 24), UNSUPPORTED), (gated(rows=1 << 40), UNSUPPORTED), (lora(rows=1 << 24), UNSUPPORTED), (norm(x=None), INVALID), (norm(y=None), INVALID), (norm(dim=0), INVALID),
    (norm(eps=0.0), INVALID), (norm(eps=float("nan")), INVALID), (norm(dim=60), UNSUPPORTED), (norm(ldx=56), INVALID),
    (norm(dim=16392, ldx=16392, ld_resid=16392, ld_sum=16392, ldy=16392), UNSUPPORTED), (norm(x_dtype=3), UNSUPPORTED),
    (norm(resid_dtype=9), UNSUPPORTED), (norm(sum_dtype=3), UNSUPPORTED), (norm(y_dtype=2), UNSUPPORTED),
    (norm(y_dtype=3), INVALID), (norm(dim=72, ldx=72, ld_resid=72, ld_sum=72, ldy=80, y_dtype=3, y_scale=at(9)), UNSUPPORTED),
    (norm(x=at(0) + 8), MISALIGNED), (norm(ldx=68), MISALIGNED), (norm(ld_resid=66), MISALIGNED), (norm(ldx=1 << 21), UNSUPPORTED),
    (norm(gamma=at(3) + 2), MISALIGNED), (norm(y_dtype=3, y_scale=at(9) + 2), MISALIGNED), (norm(y_dtype=3, y_scale=at(9), ldy=72), MISALIGNED),
    (norm(rows=4, y=at(0)), INVALID), (norm(rows=4, y=at(1) + 64), INVALID), (norm(rows=4, sum=at(0)), INVALID),
    (norm(rows=4, sum=at(1), sum_dtype=0), INVALID), (norm(rows=4, sum=at(1), ld_sum=72), INVALID), (norm(rows=4, y=at(3)), INVALID),
    (norm(rows=4, y_dtype=3, y_scale=at(0)), INVALID), (norm(rows=4, sum=at(3)), INVALID), (norm(rows=4, sum=at(1) + 16), INVALID),
    (norm_bwd(rows=-1), INVALID), (norm_bwd(s=None), INVALID), (norm_bwd(dy=None), INVALID), (norm_bwd(dx=None), INVALID),
    (norm_bwd(dim=12, ld_s=16), UNSUPPORTED), (norm_bwd(s_dtype=3), UNSUPPORTED), (norm_bwd(dx_dtype=3), UNSUPPORTED),
    (norm_bwd(dgamma=at(9)), INVALID), (norm_bwd(dgamma=at(9), workspace=at(10), workspace_bytes=255), SMALL),
    (norm_bwd(dgamma=at(9), workspace=at(10) + 4, workspace_bytes=MB), MISALIGNED), (norm_bwd(dgamma=at(9) + 4), MISALIGNED),
    (norm_bwd(rows=4, dx=at(0) + 128), INVALID), (norm_bwd(rows=4, dx=at(1), dx_dtype=2), INVALID), (norm_bwd(rows=4, dx=at(3)), INVALID),
    (norm_bwd(rows=4, dgamma=at(0), workspace=at(10), workspace_bytes=MB), INVALID),
    (norm_bwd(rows=4, dgamma=at(9), workspace=at(1), workspace_bytes=MB), INVALID), (norm_bwd(ld_dy=60), INVALID),
    (gated(rows=-3), INVALID), (gated(x=None), INVALID), (gated(gate_w=None), INVALID), (gated(up_w=None), INVALID), (gated(y=None), INVALID),
    (gated(dtype=2), UNSUPPORTED), (gated(act=2), INVALID), (gated(y_dtype=1), UNSUPPORTED), (gated(y_dtype=2), UNSUPPORTED),
    (gated(dim=60, ldx=64), UNSUPPORTED), (gated(hidden=124), UNSUPPORTED), (gated(hidden=0), INVALID), (gated(ldx=60), INVALID),
    (gated(ldx=66), MISALIGNED), (gated(ldy=120), INVALID), (gated(ldy=132), MISALIGNED), (gated(x=at(0) + 2), MISALIGNED),
    (gated(gate_w=at(1) + 8), MISALIGNED), (gated(pre=at(6) + 8), MISALIGNED), (gated(up_b=at(4) + 2), MISALIGNED),
    (gated(dim=131080, ldx=131080), UNSUPPORTED), (gated(ldx=1 << 21), UNSUPPORTED),
    (gated(rows=4, y=at(0)), INVALID), (gated(rows=4, y=at(1) + 4096), INVALID), (gated(rows=4, pre=at(5)), INVALID),
    (gated(rows=4, pre=at(2)), INVALID), (gated(rows=4, y=at(3)), INVALID),
    (gated8(pre=at(6)), UNSUPPORTED), (gated8(x_scale=None), INVALID), (gated8(gate_scale=None), INVALID), (gated8(up_scale=None), INVALID),
    (gated8(dim=72, ldx=80), UNSUPPORTED), (gated8(ldx=72), MISALIGNED), (gated8(x_scale=at(7) + 2), MISALIGNED),
    (gated8(rows=4, y=at(7)), INVALID),
    (gated_bwd(rows=-1), INVALID), (gated_bwd(dtype=3), UNSUPPORTED), (gated_bwd(dtype=2), UNSUPPORTED), (gated_bwd(act=5), INVALID),
    (gated_bwd(pre=None), INVALID), (gated_bwd(dy=None), INVALID), (gated_bwd(workspace=None), INVALID), (gated_bwd(dx=None), INVALID),
    (gated_bwd(dgate_w=at(6)), INVALID), (gated_bwd(dup_b=at(6)), INVALID), (gated_bwd(workspace_bytes=100), SMALL),
    (gated_bwd(workspace=at(10) + 16), MISALIGNED), (gated_bwd(ld_dx=60), INVALID), (gated_bwd(ld_dy=130), MISALIGNED),
    (gated_bwd(rows=4, dx=at(0)), INVALID), (gated_bwd(rows=4, dx=at(10)), INVALID), (gated_bwd(rows=4, dgate_w=at(6), dup_w=at(6)), INVALID),
    (gated_bwd(rows=4, dgate_w=at(1), dup_w=at(6)), INVALID), (gated_bwd(rows=4, dgate_b=at(6), dup_b=at(6) + 16), INVALID),
    (gated_bwd(rows=4, workspace=at(3)), INVALID),
    (lora(rows=-1), INVALID), (lora(dtype=3), UNSUPPORTED), (lora(y_dtype=2), UNSUPPORTED), (lora(rank=0), INVALID), (lora(rank=12), UNSUPPORTED),
    (lora(rank=136), UNSUPPORTED), (lora(n_adapters=-1), INVALID), (lora(a=None), INVALID), (lora(b=None), INVALID), (lora(scale=None), INVALID),
    (lora(row_adapter=None), INVALID), (lora(workspace=None), INVALID), (lora(workspace_bytes=0), SMALL), (lora(workspace=at(8) + 128), MISALIGNED),
    (lora(row_adapter=at(6) + 1), MISALIGNED), (lora(bias=at(2) + 8), MISALIGNED), (lora(dim=60, ldx=64), UNSUPPORTED),
    (lora(out_dim=132), UNSUPPORTED), (lora(ldy=120), INVALID), (lora(rows=4, y=at(0)), INVALID), (lora(rows=4, y=at(3)), INVALID),
    (lora(rows=4, workspace=at(4)), INVALID), (lora(rows=4, y=at(8)), INVALID), (lora(rows=4, workspace=at(6)), INVALID),
]


@pytest.mark.parametrize("i", range(len(REFUSED)))
def test_refusals(i):
    case, status = REFUSED[i]
    assert call(case) == status, (case[0], {n: getattr(case[1], n) for n, _ in case[1]._fields_})


def test_null_arguments():
    for n in X.EXPORTED_FFN:
        f = getattr(X.lib(), n)
        assert (f(None, None) if n.startswith("xema_op") else f(*[64] * (len(f.argtypes) - 1), None)) == INVALID, n


def test_workspace_sizes():
    # dg and du in 16 bits, 256-byte aligned, and up to 64 partial sums of 2 x hidden floats
    assert X.xema_gated_ffn_bwd_workspace_bytes(3, 64, 40) == 2 * 256 + 2 * 40 * 4
    assert X.xema_gated_ffn_bwd_workspace_bytes(100000, 4096, 4096) == 2 * 100000 * 4096 * 2 + 64 * 2 * 4096 * 4
    # and two or more fp32 sums of the weights' gradients where they have few tiles
    more = X.xema_gated_ffn_bwd_workspace_bytes(100000, 64, 4096) - (2 * 100000 * 4096 * 2 + 64 * 2 * 4096 * 4)
    assert more % (2 * 4096 * 64 * 4) == 0 and 2 <= more // (2 * 4096 * 64 * 4) <= 16
    assert X.xema_gated_ffn_pre_bytes(0, 64) == 0 and X.xema_gated_ffn_pre_bytes(100000, 4096) == 6 * 100000 * 4096
    assert X.xema_rmsnorm_bwd_workspace_bytes(1, 64) == 64 * 4
    assert X.xema_rmsnorm_bwd_workspace_bytes(100000, 64) == 1024 * 64 * 4
    assert X.xema_lora_workspace_bytes(10, 16) == 768      # two halves of 16 ranks, 16 bits each, rounded up to 256 bytes
    for f, args, status in ((X.xema_rmsnorm_bwd_workspace_bytes, (-1, 64), INVALID), (X.xema_rmsnorm_bwd_workspace_bytes, (4, 60), UNSUPPORTED),
                            (X.xema_gated_ffn_bwd_workspace_bytes, (4, 64, 0), INVALID), (X.xema_lora_workspace_bytes, (4, 12), UNSUPPORTED),
                            (X.xema_lora_workspace_bytes, (4, 0), INVALID)):
        with pytest.raises(X.XemaError) as e:
            f(*args)
        assert e.value.status == status
