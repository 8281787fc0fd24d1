"""The cross-attention sub-block's operators as timed cases: layer norm with the
residual's addition and its gradient, the linear layer with bias, activation
and residual (forward, and as a training step), and attention to an encoder's
states of another length (prompts, single tokens, and as a training step).

Token counts are those of the templates in workloads/ (two long videos of
28,612 tokens, images of 4608, a video of 17,776), odd ones and single tokens;
widths are the long-video template's 4096 and 16384 (32 heads of 128) and
generic ones; encoders have up to 512 states for prompts and up to 32,768 for
single tokens.  draw() spreads over the same ranges.
"""
import math

import torch

own = False     # whether run() calls the library, or computes the plain form

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
CODES = {"bf16": 0, "f16": 1, "f32": 2}     # xema_dtype
ACTS = {"silu": 0, "gelu": 1, "none": 2}    # xema_act
SIZE = {"bf16": 2, "f16": 2, "f32": 4, "none": 0}
EPS = 1e-6


def _ln(name, rows, dim, x, resid, out):
    return {"name": name, "kind": "ln", "rows": rows, "dim": dim, "x": x, "resid": resid, "out": out}


def _linear(name, kind, rows, dim, out, dtype, act, bias, resid, y):
    return {"name": name, "kind": kind, "rows": rows, "dim": dim, "out_dim": out, "type": dtype, "act": act, "bias": bias,
            "resid": resid, "y": y}


def _attn(name, kind, batch, heads, kv_heads, head_dim, q_len, kv_len, lens, dtype):
    return {"name": name, "kind": kind, "batch": batch, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "q_len": q_len,
            "kv_len": kv_len, "lens": lens, "type": dtype}


def listed():
    return [
        # the next token of four requests before its attention: latency
        _ln("ln_tokens", 4, 4096, "bf16", "bf16", "bf16"),
        # two long videos beside an fp32 residual stream
        _ln("ln_long", 57224, 4096, "bf16", "f32", "bf16"),
        # the gradient of a short ragged batch
        {"name": "ln_gradient_small", "kind": "ln_bwd", "rows": 1539, "dim": 2568, "type": "f16"},
        # the gradient of a training batch of eight sequences
        {"name": "ln_gradient", "kind": "ln_bwd", "rows": 16384, "dim": 4096, "type": "bf16"},
        # the output projection of the next tokens of 24 requests, onto the residual stream
        _linear("linear_tokens", "linear", 24, 4096, 4096, "bf16", "none", True, "bf16", "bf16"),
        # the output projection of two image prompts, onto an fp32 residual stream
        _linear("linear_images", "linear", 9216, 4096, 4096, "bf16", "none", True, "f32", "f32"),
        # a training step of a wide layer with its activation: the largest case
        _linear("linear_train", "linear_train", 8192, 4096, 11008, "bf16", "gelu", True, "none", "bf16"),
        # one token of each of four requests against long encodings of unlike length, four heads to one of the encoder's
        _attn("attn_tokens", "attn", 4, 32, 8, 128, 1, 16384, "ragged", "bf16"),
        # short prompts of a small model, one of them empty, odd sizes
        _attn("attn_prompts", "attn", 3, 12, 12, 72, 333, 77, "empty", "f16"),
        # two long videos against their prompts
        _attn("attn_videos", "attn", 2, 32, 32, 128, 28612, 512, "ragged", "bf16"),
        # a training step of a small layer on ragged prompts, heads shared
        _attn("attn_train_small", "attn_train", 3, 16, 4, 72, 577, 120, "ragged", "f16"),
        # a training step on two image sequences
        _attn("attn_train_images", "attn_train", 2, 32, 32, 128, 4608, 512, "full", "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A multiple of 8: half of the draws from 512 on a multiple of 256."""
    w = _log(rng, lo, hi)
    return w // 256 * 256 if w >= 512 and rng.random() < 0.5 else (w + 7) // 8 * 8


def draw(rng):
    most_products = 0.8 * 6 * 8192 * 4096 * 11008
    kind = rng.choice(("ln", "ln_bwd", "linear", "linear_train", "attn", "attn", "attn_token", "attn_train", "attn_train"))
    while True:
        if kind == "ln":
            c = _ln("", _log(rng, 1, 57000), _width(rng, 256, 8192), rng.choice(("bf16", "f16", "f32")),
                    rng.choice(("none", "bf16", "f16", "f32")), rng.choice(("bf16", "f16", "f32")))
            fits = c["rows"] * c["dim"] <= 57224 * 4096
        elif kind == "ln_bwd":
            c = {"name": "", "kind": kind, "rows": _log(rng, 1, 40000), "dim": _width(rng, 256, 8192), "type": rng.choice(("bf16", "f16"))}
            fits = c["rows"] * c["dim"] <= 16384 * 4096
        elif kind in ("linear", "linear_train"):
            dtype, train = rng.choice(("bf16", "f16")), kind == "linear_train"
            c = _linear("", kind, _log(rng, 1, 20000), _width(rng, 256, 6144), _width(rng, 256, 16384), dtype,
                        rng.choice(("none", "silu", "gelu")), rng.choice((False, True)),
                        "none" if train else rng.choice(("none", "bf16", "f16", "f32")), dtype if train else rng.choice((dtype, "f32")))
            fits = work(c)["flops"] <= most_products
        else:
            kv_heads, group, dtype = rng.randint(1, 32), rng.choice((1, 1, 1, 2, 4, 8)), rng.choice(("bf16", "f16"))
            d = rng.choice((64, 128, 64, 128, 8 * rng.randint(4, 16)))
            lens = rng.choice(("full", "ragged", "ragged", "empty"))
            token = kind == "attn_token"
            q_len = rng.choice((1, 1, rng.randint(2, 16))) if token else _log(rng, 16, 28612)
            kv_len = _log(rng, 64, 32768) if token else _log(rng, 8, 1024)
            c = _attn("", "attn" if token else kind, rng.randint(1, 8), kv_heads * group, kv_heads, d, q_len, kv_len, lens, dtype)
            scores = c["batch"] * c["heads"] * q_len * kv_len
            fits = (scores <= 0.8 * 2 * 32 * (4608 if kind == "attn_train" else 28612) * 512
                    and c["batch"] * c["heads"] * d * q_len <= 2 * 4096 * (14306 if kind == "attn_train" else 28612)
                    and c["batch"] * kv_heads * d * kv_len <= 4 * 1024 * 16384)
        if fits:
            del c["name"]
            return c


# -- inputs ------------------------------------------------------------------------------------------------------


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(g, shape, std=1.0, dtype=torch.bfloat16, mean=0.0):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).mul_(std).add_(mean).to(dtype)


def _lens(c):
    """Encoder states of each sequence: all of them, unlike numbers, or unlike numbers with the last sequence empty."""
    n, b = c["kv_len"], c["batch"]
    if c["lens"] == "full":
        return [n] * b
    lens = [max(1, n * (b - i) // b) for i in range(b)]
    return lens[:-1] + [0] if c["lens"] == "empty" and b > 1 else lens


def _ln_inputs(c, seed):
    g, shape = _gen(seed), (c["rows"], c["dim"])
    # tokens of unlike sizes and means, as a residual stream holds them, and a few large channels
    size = torch.exp(torch.randn((c["rows"], 1), generator=g, device=DEV))
    mean = torch.randn((c["rows"], 1), generator=g, device=DEV)
    big = 1 + 7 * (torch.rand((1, c["dim"]), generator=g, device=DEV) < 0.01)
    d = {"x": (_normal(g, shape, dtype=torch.float32) * big + mean).to(TYPES[c["x"]]),
         "gamma": _normal(g, (c["dim"],), 0.1, mean=1.0), "beta": _normal(g, (c["dim"],), 0.1)}
    if c["resid"] != "none":
        d["resid"] = (_normal(g, shape, dtype=torch.float32) * size).to(TYPES[c["resid"]])
    return d


def _ln_bwd_inputs(c, seed):
    g, shape, t = _gen(seed), (c["rows"], c["dim"]), TYPES[c["type"]]
    return {"x": _normal(g, shape, 2.0, t, 0.5), "dy": _normal(g, shape, 1e-2, t), "dsum": _normal(g, shape, 1e-2, t),
            "gamma": _normal(g, (c["dim"],), 0.1, mean=1.0)}


def _linear_inputs(c, seed):
    g, M, D, N, t = _gen(seed), c["rows"], c["dim"], c["out_dim"], TYPES[c["type"]]
    d = {"x": _normal(g, (M, D), dtype=t), "w": _normal(g, (N, D), D ** -0.5, t)}
    if c["bias"]:
        d["bias"] = _normal(g, (N,), 0.5)
    if c["resid"] != "none":
        d["resid"] = _normal(g, (M, N), 2.0, TYPES[c["resid"]])
    if c["kind"] == "linear_train":
        d["dy"] = _normal(g, (M, N), 0.05, t)
    return d


def _attn_inputs(c, seed):
    g, t = _gen(seed), TYPES[c["type"]]
    B, H, KH, d, Lq, S = (c[k] for k in ("batch", "heads", "kv_heads", "head_dim", "q_len", "kv_len"))
    # keys and values come side by side from one projection; every sequence's first state draws more weight than the others
    kv = _normal(g, (B, S, 2, KH, d), 1.0, torch.float32)
    q = _normal(g, (B, Lq, H, d), 1.5, torch.float32)
    kv[:, 0, 0] += 0.5
    q += 0.25
    st = {"q": q.to(t).view(B * Lq, H * d), "kv": kv.to(t).view(B * S, 2 * KH * d),
          "lens": torch.tensor(_lens(c), dtype=torch.int32, device=DEV)}
    if c["kind"] == "attn_train":
        st["do"] = _normal(g, (B * Lq, H * d), 0.05, t)
    return st


INPUTS = {"ln": _ln_inputs, "ln_bwd": _ln_bwd_inputs, "linear": _linear_inputs, "linear_train": _linear_inputs, "attn": _attn_inputs,
          "attn_train": _attn_inputs}


def prepare(case, seed):
    """The inputs and the buffers that a program allocates once."""
    c = case
    st = dict(INPUTS[c["kind"]](c, seed), case=c)
    if c["kind"] == "ln":
        shape = (c["rows"], c["dim"])
        st["y"] = torch.empty(shape, dtype=TYPES[c["out"]], device=DEV)
        if c["resid"] != "none":
            st["sum"] = torch.empty(shape, dtype=TYPES[c["resid"]], device=DEV)
    elif c["kind"] == "ln_bwd":
        st["dx"] = torch.empty_like(st["x"])
        st["dgamma"], st["dbeta"] = (torch.empty(c["dim"], dtype=torch.float32, device=DEV) for _ in range(2))
    elif c["kind"] in ("linear", "linear_train"):
        st["y"] = torch.empty((c["rows"], c["out_dim"]), dtype=TYPES[c["y"]], device=DEV)
        if c["kind"] == "linear_train":
            if c["act"] != "none":
                st["pre"] = torch.empty(3 * c["rows"] * c["out_dim"], dtype=torch.uint8, device=DEV)   # z in 24 bits
            for n in ("x", "w") + (("bias",) if c["bias"] else ()):
                st["d" + n] = torch.empty_like(st[n])
    else:
        st["o"] = torch.empty_like(st["q"])
        if c["kind"] == "attn_train":
            st["lse"] = torch.empty((c["batch"], c["heads"], c["q_len"]), dtype=torch.float32, device=DEV)
            st["dq"], st["dkv"] = torch.empty_like(st["q"]), torch.empty_like(st["kv"])
    return st


# -- the calls ---------------------------------------------------------------------------------------------------


def _workspace(st, nbytes):
    """A program's scratch memory, allocated once."""
    if st.get("ws") is None:
        st["ws"] = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=DEV)
    return st["ws"]


def _calls(X, st):
    """The calls of one pass, their arguments laid out once: (entry point, arguments) pairs, and the outputs."""
    c, t = st["case"], CODES.get(st["case"].get("type"), 0)
    if c["kind"] == "ln":
        a = X.layernorm_args(st["x"], CODES[c["x"]], c["rows"], c["dim"], st["gamma"], st["beta"], EPS, st["y"], CODES[c["out"]],
                             resid=st.get("resid"), resid_dtype=CODES.get(c["resid"], 0), sum=st.get("sum"),
                             sum_dtype=CODES.get(c["resid"], 0))
        return [(X.xema_op_layernorm, a)], {k: st[k] for k in ("y", "sum") if k in st}
    if c["kind"] == "ln_bwd":
        ws = _workspace(st, X.xema_layernorm_bwd_workspace_bytes(c["rows"], c["dim"]))
        a = X.layernorm_bwd_args(st["x"], t, c["rows"], c["dim"], st["gamma"], EPS, st["dy"], t, st["dx"], t, st["dgamma"], st["dbeta"],
                                 ws, ws.numel(), dsum=st["dsum"], dsum_dtype=t)
        return [(X.xema_op_layernorm_bwd, a)], {k: st[k] for k in ("dx", "dgamma", "dbeta")}
    if c["kind"] in ("linear", "linear_train"):
        M, D, N, act = c["rows"], c["dim"], c["out_dim"], ACTS[c["act"]]
        calls = [(X.xema_op_linear, X.linear_args(t, st["x"], M, D, st["w"], N, st.get("bias"), act, st["y"], CODES[c["y"]],
                                                  resid=st.get("resid"), resid_dtype=CODES.get(c["resid"], 0), pre=st.get("pre")))]
        if c["kind"] == "linear":
            return calls, st["y"]
        ws = _workspace(st, X.xema_linear_bwd_workspace_bytes(M, D, N))
        calls.append((X.xema_op_linear_bwd, X.linear_bwd_args(t, act, st["x"], M, D, st["w"], N, st.get("pre"), st["dy"], t, st["dx"],
                                                              st["dw"], st.get("dbias"), ws, ws.numel())))
        return calls, {k: st[k] for k in ("y", "dx", "dw", "dbias") if k in st}
    sizes = tuple(c[k] for k in ("batch", "heads", "kv_heads", "head_dim", "q_len", "kv_len"))
    n, scale = c["kv_heads"] * c["head_dim"], c["head_dim"] ** -0.5
    k, v = st["kv"][:, :n], st["kv"][:, n:]
    train = c["kind"] == "attn_train"
    need = X.xema_cross_attn_workspace_bytes(*sizes)
    if train:
        need = max(need, X.xema_cross_attn_bwd_workspace_bytes(*sizes))
    ws = _workspace(st, need)
    calls = [(X.xema_op_cross_attn, X.cross_attn_args(t, *sizes, st["q"], k, v, scale, st["o"], ws, ws.numel(), lse=st.get("lse"),
                                                      kv_lens=st["lens"], ldk=2 * n, ldv=2 * n))]
    if not train:
        return calls, st["o"]
    dk, dv = st["dkv"][:, :n], st["dkv"][:, n:]
    calls.append((X.xema_op_cross_attn_bwd, X.cross_attn_bwd_args(t, *sizes, st["q"], k, v, scale, st["o"], st["lse"], st["do"], st["dq"],
                                                                  dk, dv, ws, ws.numel(), kv_lens=st["lens"], ldk=2 * n, ldv=2 * n,
                                                                  ld_dk=2 * n, ld_dv=2 * n)))
    return calls, {k: st[k] for k in ("o", "dq", "dkv")}


def _own(st):
    import paper_2607_11136_amd as X
    if "calls" not in st:
        st["calls"] = _calls(X, st)
    calls, outputs = st["calls"]
    for call, args in calls:
        call(args)
    return outputs


def _act(z, name):
    """(act(z), act'(z))"""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    a = math.sqrt(2 / math.pi)
    th = torch.tanh(a * (z + 0.044715 * z * z * z))
    return 0.5 * z * (1 + th), 0.5 * (1 + th) + 0.5 * z * (1 - th * th) * a * (1 + 3 * 0.044715 * z * z)


def _plain(st):
    c = st["case"]
    if c["kind"] == "ln":
        s = st["x"].float()
        if "resid" in st:
            s = s + st["resid"].float()
        e = s - s.mean(1, keepdim=True)
        y = e * torch.rsqrt((e * e).mean(1, keepdim=True) + EPS) * st["gamma"].float() + st["beta"].float()
        return {"y": y.to(st["y"].dtype), **({"sum": s.to(st["sum"].dtype)} if "sum" in st else {})}
    if c["kind"] == "ln_bwd":
        x, dy = st["x"].float(), st["dy"].float()
        e = x - x.mean(1, keepdim=True)
        q = torch.rsqrt((e * e).mean(1, keepdim=True) + EPS)
        n, g = e * q, dy * st["gamma"].float()
        dx = q * (g - g.mean(1, keepdim=True) - n * (g * n).mean(1, keepdim=True)) + st["dsum"].float()
        return {"dx": dx.to(st["dx"].dtype), "dgamma": (dy * n).sum(0), "dbeta": dy.sum(0)}
    if c["kind"] in ("linear", "linear_train"):
        x, w = st["x"].float(), st["w"].float()
        z = x @ w.t()
        if c["bias"]:
            z = z + st["bias"].float()
        a, da = _act(z, c["act"])
        y = (a + st["resid"].float() if "resid" in st else a).to(st["y"].dtype)
        if c["kind"] == "linear":
            return y
        dz, t = st["dy"].float() * da, st["x"].dtype
        return {"y": y, "dx": (dz @ w).to(t), "dw": (dz.t() @ x).to(t), **({"dbias": dz.sum(0).bfloat16()} if c["bias"] else {})}
    B, H, KH, d, Lq, S = (c[k] for k in ("batch", "heads", "kv_heads", "head_dim", "q_len", "kv_len"))
    t, scale = st["q"].dtype, d ** -0.5
    # [batch, kv head, query (its heads side by side), d] and [batch, kv head, state, d]
    G = H // KH

    def by_head(x):
        return x.float().view(B, Lq, KH, G, d).permute(0, 2, 1, 3, 4).reshape(B, KH, Lq * G, d)

    def from_heads(x):
        return x.view(B, KH, Lq, G, d).permute(0, 2, 1, 3, 4).reshape(B * Lq, H * d).to(t)

    q = by_head(st["q"])
    k, v = st["kv"].float().view(B, S, 2, KH, d).permute(2, 0, 3, 1, 4).contiguous()
    there = (torch.arange(S, device=DEV)[None] < st["lens"][:, None]).view(B, 1, 1, S)
    s = torch.where(there, q @ k.transpose(2, 3).contiguous() * scale, -math.inf)
    m = s.amax(3, keepdim=True).clamp(min=-1e30)
    e = torch.exp(s - m)
    p = e / e.sum(3, keepdim=True).clamp(min=1e-30)
    o = p @ v
    if c["kind"] == "attn":
        return from_heads(o)
    do = by_head(st["do"])
    dp = do @ v.transpose(2, 3).contiguous()
    ds = p * (dp - (do * o).sum(3, keepdim=True)) * scale
    dk, dv = ds.transpose(2, 3).contiguous() @ q, p.transpose(2, 3).contiguous() @ do
    dkv = torch.stack((dk, dv)).permute(1, 3, 0, 2, 4).reshape(B * S, 2 * KH * d)
    return {"o": from_heads(o), "dq": from_heads(ds @ k), "dkv": dkv.to(t)}


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    c = case
    if c["kind"] == "ln":
        n = c["rows"] * c["dim"]
        return {"bytes": n * (SIZE[c["x"]] + 2 * SIZE[c["resid"]] + SIZE[c["out"]]) + 4 * c["dim"], "flops": 8 * n}
    if c["kind"] == "ln_bwd":
        n = c["rows"] * c["dim"]
        return {"bytes": 8 * n + 10 * c["dim"], "flops": 16 * n}
    if c["kind"] in ("linear", "linear_train"):
        M, D, N = c["rows"], c["dim"], c["out_dim"]
        if c["kind"] == "linear":
            return {"bytes": 2 * (M * D + N * D) + M * N * (SIZE[c["resid"]] + SIZE[c["y"]]), "flops": 2 * M * N * D}
        return {"bytes": 2 * (2 * M * D + 2 * M * N + 2 * N * D), "flops": 6 * M * N * D}
    states, d, train = sum(_lens(c)), c["head_dim"], c["kind"] == "attn_train"
    products = 2 * c["q_len"] * states * c["heads"] * d
    rows = c["batch"] * c["q_len"] * c["heads"] * d
    # forward: q, k, v, o; a training step: do, dq and the gradients of all states too
    kv = 2 * states * c["kv_heads"] * d + (2 * c["batch"] * c["kv_len"] * c["kv_heads"] * d if train else 0)
    return {"bytes": 2 * ((4 if train else 2) * rows + kv), "flops": (7 if train else 2) * products}


# -- the same in 64 bits -----------------------------------------------------------------------------------------


def exact(case, seed):
    c = case
    d = INPUTS[c["kind"]](c, seed)
    if c["kind"] in ("ln", "ln_bwd"):
        z = {k: v.double() for k, v in d.items()}
        s = z["x"] + z["resid"] if "resid" in z else z["x"]
        mean, var = s.mean(1, keepdim=True), s.var(1, unbiased=False, keepdim=True)
        std = torch.sqrt(var + EPS)
        if c["kind"] == "ln":
            y = torch.addcmul(z["beta"], (s - mean) / std, z["gamma"])
            return {"y": y, **({"sum": s} if "resid" in z else {})}
        # dy_i/dx_j = gamma_i / std (delta_ij - 1/n - (x_i - mean)(x_j - mean) / (n std^2))
        e, g, n = s - mean, z["dy"] * z["gamma"], c["dim"]
        dx = g / std - g.sum(1, keepdim=True) / (n * std) - e * (g * e).sum(1, keepdim=True) / (n * std ** 3) + z["dsum"]
        return {"dx": dx, "dgamma": (z["dy"] * e / std).sum(0), "dbeta": z["dy"].sum(0)}
    if c["kind"] in ("linear", "linear_train"):
        z = {k: v.double() for k, v in d.items()}
        pre = torch.nn.functional.linear(z["x"], z["w"], z.get("bias"))
        if c["act"] == "silu":
            e = torch.exp(-pre)
            act, slope = pre / (1 + e), torch.where(pre < -300, 0.0, (1 + e + pre * e) / (1 + e) ** 2)
        elif c["act"] == "gelu":
            k = math.sqrt(8 / math.pi)     # (1 + tanh(z)) / 2 = 1 / (1 + exp(-2 z))
            p = 1 / (1 + torch.exp(-k * (pre + 0.044715 * pre ** 3)))
            act, slope = pre * p, p + pre * p * (1 - p) * k * (1 + 0.134145 * pre ** 2)
        else:
            act, slope = pre, 1.0
        y = act + z["resid"] if "resid" in z else act
        if c["kind"] == "linear":
            return y
        dz = z["dy"] * slope
        return {"y": y, "dx": dz @ z["w"], "dw": dz.t().contiguous() @ z["x"], **({"dbias": dz.sum(0)} if c["bias"] else {})}
    B, H, KH, w, Lq, S = (c[k] for k in ("batch", "heads", "kv_heads", "head_dim", "q_len", "kv_len"))
    train = c["kind"] == "attn_train"
    q = d["q"].view(B, Lq, H, w)
    k, v = d["kv"].view(B, S, 2, KH, w).unbind(2)
    do = d["do"].view(B, Lq, H, w) if train else None
    o = torch.zeros((B, Lq, H, w), dtype=torch.float64, device=DEV)
    dq, dkv = torch.zeros_like(o), torch.zeros((B, S, 2, KH, w), dtype=torch.float64, device=DEV)
    for b, n in enumerate(_lens(c)):      # one sequence, its own states alone, one head at a time
        for h in range(H if n else 0):
            g = h * KH // H
            qh, kh, vh = q[b, :, h].double(), k[b, :n, g].double(), v[b, :n, g].double()
            p = torch.softmax(qh @ kh.t() / math.sqrt(w), 1)
            o[b, :, h] = p @ vh
            if train:
                dh = do[b, :, h].double()
                dp = dh @ vh.t()
                ds = p * (dp - (p * dp).sum(1, keepdim=True)) / math.sqrt(w)
                dq[b, :, h] = ds @ kh
                dkv[b, :n, 0, g] += ds.t() @ qh
                dkv[b, :n, 1, g] += p.t() @ dh
    o = o.view(B * Lq, H * w)
    return {"o": o, "dq": dq.view(B * Lq, H * w), "dkv": dkv.view(B * S, 2 * KH * w)} if train else o
