"""The cross-attention sub-block's entry points without a GPU: exports, struct
layouts, the documented refusals (all before any device work), workspace sizes."""
import ctypes
import os
import re

import pytest

import paper_2607_11136_amd as X

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED, SMALL, MISALIGNED = (X.XEMA_ERR_INVALID_ARG, X.XEMA_ERR_UNSUPPORTED, X.XEMA_ERR_WORKSPACE_TOO_SMALL,
                                           X.XEMA_ERR_MISALIGNED)
BIG = 1 << 31


def test_exports_are_those_of_the_header():
    src = open(os.path.join(ROOT, "include", "xema_cross.h")).read()
    names = set(re.findall(r"XEMA_API\s+[\w\s\*]+?\b(xema_\w+)\s*\(", src))
    assert names == set(X.EXPORTED_CROSS) and not names & (set(X.EXPORTED) | set(X.EXPORTED_FFN))
    for n in names:
        assert hasattr(X.lib(), n), n


def test_structs_have_the_headers_fields():
    src = open(os.path.join(ROOT, "include", "xema_cross.h")).read()
    for name, cls in (("xema_layernorm_args", X.LayernormArgs), ("xema_layernorm_bwd_args", X.LayernormBwdArgs), ("xema_linear_args", X.LinearArgs),
                      ("xema_linear_bwd_args", X.LinearBwdArgs), ("xema_cross_attn_args", X.CrossAttnArgs),
                      ("xema_cross_attn_bwd_args", X.CrossAttnBwdArgs)):
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
             gamma=at(3), beta=at(5), eps=1e-6, y=at(4), y_dtype=0, ldy=64)
    a.update(kw)
    return "xema_op_layernorm", X.LayernormArgs(**a)


def norm_bwd(**kw):
    a = dict(rows=0, dim=64, s=at(0), s_dtype=0, ld_s=64, dy=at(1), dy_dtype=0, ld_dy=64, dsum=at(2), dsum_dtype=0, ld_dsum=64, gamma=at(3),
             eps=1e-6, dx=at(4), dx_dtype=0, ld_dx=64, dgamma=None, dbeta=None, workspace=None, workspace_bytes=0)
    a.update(kw)
    return "xema_op_layernorm_bwd", X.LayernormBwdArgs(**a)


def linear(**kw):
    a = dict(dtype=0, act=2, rows=0, dim=64, out_dim=128, x=at(0), ldx=64, w=at(1), bias=at(2), resid=at(3), resid_dtype=2, ld_resid=128, y=at(4),
             y_dtype=2, ldy=128, pre=at(5))
    a.update(kw)
    return "xema_op_linear", X.LinearArgs(**a)


def linear_bwd(**kw):
    a = dict(dtype=0, act=1, rows=0, dim=64, out_dim=128, x=at(0), ldx=64, w=at(1), pre=at(2), dy=at(3), dy_dtype=0, ld_dy=128, dx=at(4), ld_dx=64,
             dw=None, dbias=None, workspace=at(10), workspace_bytes=BIG)
    a.update(kw)
    return "xema_op_linear_bwd", X.LinearBwdArgs(**a)


def attn(**kw):
    a = dict(dtype=0, batch=2, heads=4, kv_heads=2, head_dim=64, q_len=0, kv_len=10, q=at(0), ldq=256, k=at(1), ldk=128, v=at(2), ldv=128,
             kv_lens=at(3), scale=0.125, o=at(4), ldo=256, lse=at(5), workspace=at(10), workspace_bytes=BIG)
    a.update(kw)
    return "xema_op_cross_attn", X.CrossAttnArgs(**a)


def attn_bwd(**kw):
    a = dict(dtype=0, batch=2, heads=4, kv_heads=2, head_dim=64, q_len=0, kv_len=0, q=at(0), ldq=256, k=at(1), ldk=128, v=at(2), ldv=128,
             kv_lens=at(3), scale=0.125, o=at(4), ldo=256, lse=at(5), dout=at(6), ld_do=256, dq=at(7), ld_dq=256, dk=at(8), ld_dk=128, dv=at(9),
             ld_dv=128, workspace=at(10), workspace_bytes=BIG)
    a.update(kw)
    return "xema_op_cross_attn_bwd", X.CrossAttnBwdArgs(**a)


def call(case):
    return getattr(X.lib(), case[0])(ctypes.byref(case[1]), None)


@pytest.mark.parametrize("case", [norm(), norm(resid=None, sum=None, gamma=None, beta=None), norm(y_dtype=2), norm(sum=at(1)), norm_bwd(),
                                  norm_bwd(dsum=None), linear(), linear(bias=None, resid=None, pre=None, act=0), linear(y=at(3)), linear_bwd(),
                                  linear_bwd(act=2, pre=None, dy_dtype=2), attn(), attn(batch=0), attn(lse=None, kv_lens=None, workspace=None),
                                  attn_bwd(), attn_bwd(dq=None), attn_bwd(dk=None, dv=None)], ids=lambda c: c[0])
def test_empty_calls_are_taken(case):
    assert call(case) == X.XEMA_OK


Q = dict(q_len=3)
REFUSED = [
    (norm(rows=-1), INVALID), (norm(rows=1 << 24), UNSUPPORTED), (norm(x=None), INVALID), (norm(y=None), INVALID), (norm(dim=0), INVALID),
    (norm(eps=0.0), INVALID), (norm(eps=float("nan")), INVALID), (norm(dim=60), UNSUPPORTED), (norm(ldx=56), INVALID),
    (norm(dim=16392, ldx=16392, ld_resid=16392, ld_sum=16392, ldy=16392), UNSUPPORTED), (norm(x_dtype=3), UNSUPPORTED),
    (norm(resid_dtype=9), UNSUPPORTED), (norm(sum_dtype=3), UNSUPPORTED), (norm(y_dtype=3), UNSUPPORTED), (norm(x=at(0) + 8), MISALIGNED),
    (norm(ldx=68), MISALIGNED), (norm(ld_resid=66), MISALIGNED), (norm(ldx=1 << 21), UNSUPPORTED), (norm(gamma=at(3) + 2), MISALIGNED),
    (norm(beta=at(5) + 8), MISALIGNED), (norm(rows=4, y=at(0)), INVALID), (norm(rows=4, y=at(1) + 64), INVALID), (norm(rows=4, sum=at(0)), INVALID),
    (norm(rows=4, sum=at(1), sum_dtype=0), INVALID), (norm(rows=4, sum=at(1), ld_sum=72), INVALID), (norm(rows=4, y=at(5)), INVALID),
    (norm(rows=4, sum=at(3)), INVALID), (norm(rows=4, sum=at(1) + 16), INVALID),
    (norm_bwd(rows=-1), INVALID), (norm_bwd(s=None), INVALID), (norm_bwd(dy=None), INVALID), (norm_bwd(dx=None), INVALID),
    (norm_bwd(dim=12, ld_s=16), UNSUPPORTED), (norm_bwd(s_dtype=3), UNSUPPORTED), (norm_bwd(dx_dtype=3), UNSUPPORTED),
    (norm_bwd(dgamma=at(9)), INVALID), (norm_bwd(dbeta=at(9)), INVALID), (norm_bwd(dbeta=at(9), workspace=at(10), workspace_bytes=511), SMALL),
    (norm_bwd(dgamma=at(9), workspace=at(10) + 4, workspace_bytes=BIG), MISALIGNED), (norm_bwd(dbeta=at(9) + 4), MISALIGNED),
    (norm_bwd(rows=4, dx=at(0) + 128), INVALID), (norm_bwd(rows=4, dx=at(1), dx_dtype=2), INVALID), (norm_bwd(rows=4, dx=at(3)), INVALID),
    (norm_bwd(rows=4, dgamma=at(9), dbeta=at(9), workspace=at(10), workspace_bytes=BIG), INVALID),
    (norm_bwd(rows=4, dbeta=at(0), workspace=at(10), workspace_bytes=BIG), INVALID),
    (norm_bwd(rows=4, dbeta=at(9), workspace=at(1), workspace_bytes=BIG), INVALID), (norm_bwd(ld_dy=60), INVALID),
    (linear(rows=-1), INVALID), (linear(rows=1 << 24), UNSUPPORTED), (linear(x=None), INVALID), (linear(w=None), INVALID), (linear(y=None), INVALID),
    (linear(act=3), INVALID), (linear(act=-1), INVALID), (linear(dtype=2), UNSUPPORTED), (linear(dtype=3), UNSUPPORTED), (linear(y_dtype=3), UNSUPPORTED),
    (linear(resid_dtype=3), UNSUPPORTED), (linear(dim=60, ldx=64), UNSUPPORTED), (linear(out_dim=132), UNSUPPORTED), (linear(out_dim=0), INVALID),
    (linear(ldx=56), INVALID), (linear(ldy=130), MISALIGNED), (linear(ld_resid=120), INVALID), (linear(bias=at(2) + 8), MISALIGNED),
    (linear(pre=at(5) + 8), MISALIGNED), (linear(w=at(1) + 8), MISALIGNED), (linear(rows=4, y=at(0)), INVALID), (linear(rows=4, y=at(1)), INVALID),
    (linear(rows=4, y=at(3), y_dtype=0), INVALID), (linear(rows=4, y=at(3) + 16), INVALID), (linear(rows=4, pre=at(4)), INVALID),
    (linear(rows=4, pre=at(3)), INVALID), (linear(rows=4, y=at(2)), INVALID), (linear(ldy=1 << 21), UNSUPPORTED),
    (linear_bwd(rows=-1), INVALID), (linear_bwd(act=4), INVALID), (linear_bwd(pre=None), INVALID), (linear_bwd(dx=None), INVALID),
    (linear_bwd(workspace=None), INVALID), (linear_bwd(workspace_bytes=100), SMALL), (linear_bwd(workspace=at(10) + 16), MISALIGNED),
    (linear_bwd(dy_dtype=1), UNSUPPORTED), (linear_bwd(dtype=2), UNSUPPORTED), (linear_bwd(ld_dx=60), INVALID), (linear_bwd(ld_dy=132), MISALIGNED),
    (linear_bwd(dbias=at(6) + 2), MISALIGNED), (linear_bwd(rows=4, dx=at(0)), INVALID), (linear_bwd(rows=4, dx=at(3)), INVALID),
    (linear_bwd(rows=4, dx=at(10)), INVALID), (linear_bwd(rows=4, dw=at(1)), INVALID), (linear_bwd(rows=4, dw=at(6), dbias=at(6)), INVALID),
    (linear_bwd(rows=4, workspace=at(2)), INVALID),
    (attn(batch=-1), INVALID), (attn(q_len=-1), INVALID), (attn(kv_len=-1), INVALID), (attn(heads=0), INVALID), (attn(kv_heads=0), INVALID),
    (attn(kv_heads=3), INVALID), (attn(head_dim=0), INVALID), (attn(head_dim=60), UNSUPPORTED), (attn(head_dim=136), UNSUPPORTED), (attn(dtype=2), UNSUPPORTED),
    (attn(scale=0.0), INVALID), (attn(scale=-1.0), INVALID), (attn(scale=float("nan")), INVALID), (attn(scale=float("inf")), INVALID),
    (attn(q=None), INVALID), (attn(k=None), INVALID), (attn(v=None), INVALID), (attn(o=None), INVALID), (attn(ldq=248), INVALID), (attn(ldk=130), MISALIGNED),
    (attn(ldv=1 << 21), UNSUPPORTED), (attn(o=at(4) + 8), MISALIGNED), (attn(kv_lens=at(3) + 2), MISALIGNED), (attn(lse=at(5) + 1), MISALIGNED),
    (attn(workspace=at(10) + 16), MISALIGNED), (attn(q_len=1 << 23), UNSUPPORTED), (attn(kv_len=1 << 24), UNSUPPORTED),
    (attn(heads=4096, ldq=1 << 18, ldo=1 << 18), UNSUPPORTED),
    (attn(batch=1 << 21, q_len=1, heads=4), UNSUPPORTED), (attn(**Q, o=at(0)), INVALID), (attn(**Q, o=at(1) + 256), INVALID), (attn(**Q, o=at(5)), INVALID),
    (attn(**Q, lse=at(2)), INVALID), (attn(**Q, o=at(3)), INVALID), (attn(batch=1, q_len=1, kv_len=20000, workspace=None), INVALID),
    (attn(batch=1, q_len=1, kv_len=20000, workspace_bytes=1000), SMALL), (attn(batch=1, q_len=1, kv_len=20000, workspace=at(4)), INVALID),
    (attn_bwd(dq=None, dk=None, dv=None), INVALID), (attn_bwd(dk=None), INVALID), (attn_bwd(dv=None), INVALID), (attn_bwd(lse=None), INVALID),
    (attn_bwd(o=None), INVALID), (attn_bwd(dout=None), INVALID), (attn_bwd(workspace=None), INVALID), (attn_bwd(**Q, workspace_bytes=10), SMALL),
    (attn_bwd(workspace=at(10) + 64), MISALIGNED), (attn_bwd(ld_dq=200), INVALID), (attn_bwd(ld_dk=132), MISALIGNED), (attn_bwd(scale=0.0), INVALID),
    (attn_bwd(head_dim=12), UNSUPPORTED), (attn_bwd(**Q, dq=at(0)), INVALID), (attn_bwd(**Q, dq=at(6)), INVALID), (attn_bwd(kv_len=5, dk=at(1)), INVALID),
    (attn_bwd(kv_len=5, dv=at(8)), INVALID), (attn_bwd(**Q, dq=at(10)), INVALID), (attn_bwd(**Q, workspace=at(5)), INVALID),
]


@pytest.mark.parametrize("i", range(len(REFUSED)))
def test_refusals(i):
    case, status = REFUSED[i]
    assert call(case) == status, (case[0], {n: getattr(case[1], n) for n, _ in case[1]._fields_})


def test_null_arguments():
    for n in X.EXPORTED_CROSS:
        f = getattr(X.lib(), n)
        assert (f(None, None) if n.startswith("xema_op") else f(*[64] * (len(f.argtypes) - 1), None)) == INVALID, n


def test_workspace_sizes():
    assert X.xema_layernorm_bwd_workspace_bytes(1, 64) == 2 * 64 * 4
    assert X.xema_layernorm_bwd_workspace_bytes(100000, 64) == 512 * 2 * 64 * 4
    assert X.xema_linear_pre_bytes(0, 64) == 0 and X.xema_linear_pre_bytes(100000, 4096) == 3 * 100000 * 4096
    # dz in 16 bits, and up to 64 partial sums of out_dim floats
    assert X.xema_linear_bwd_workspace_bytes(3, 64, 40) == 256 + 40 * 4
    assert X.xema_linear_bwd_workspace_bytes(100000, 4096, 4096) == 100000 * 4096 * 2 + 64 * 4096 * 4
    assert X.xema_cross_attn_workspace_bytes(2, 32, 32, 128, 28612, 512) == 0
    # one token: parts of o, each with a maximum and a sum
    n = X.xema_cross_attn_workspace_bytes(1, 32, 8, 128, 1, 16384)
    assert n % (32 * (128 * 4 + 8)) == 0 and 2 <= n // (32 * (128 * 4 + 8)) <= 64
    # lse and D of every token and head
    assert X.xema_cross_attn_bwd_workspace_bytes(2, 32, 32, 128, 28612, 512) % 8 == 0
    assert X.xema_cross_attn_bwd_workspace_bytes(2, 32, 32, 128, 28612, 512) >= 2 * 2 * 32 * 28612 * 4
    for f, args, status in ((X.xema_layernorm_bwd_workspace_bytes, (-1, 64), INVALID), (X.xema_linear_pre_bytes, (4, 60), UNSUPPORTED),
                            (X.xema_linear_bwd_workspace_bytes, (4, 64, 0), INVALID), (X.xema_cross_attn_workspace_bytes, (1, 4, 3, 64, 1, 1), INVALID),
                            (X.xema_cross_attn_bwd_workspace_bytes, (1, 4, 2, 68, 1, 1), UNSUPPORTED)):
        with pytest.raises(X.XemaError) as e:
            f(*args)
        assert e.value.status == status
