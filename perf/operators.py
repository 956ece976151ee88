"""Operators of a transformer block as cases to measure: layer norm with modulation and its backward pass, rotary
positions with several axes and their inverse, and the gated linear layer (both projections, activation, product)
with its backward pass.

`run` computes a case either in its plain form, with elementary torch operations in 32 bits, or (where `own` is true)
with this framework's operators; `exact` gives the same outputs from the definitions in 64 bits.
"""
import math

import torch

own = False

_T = {"bf16": torch.bfloat16, "fp32": torch.float32}
_BYTES = {"bf16": 2, "fp32": 4}


# ------------------------------------------------------------------------------------------------ cases
def _norm(name, back, groups, rows, D, x, y, weight="unit"):
    # weight: "unit" = 1 + scale per group (adaptive norm), "plain" = a learned weight and bias, "none" = neither
    c = {"op": "norm_bwd" if back else "norm", "groups": groups, "rows": rows, "D": D, "x": x, "y": y, "weight": weight}
    return {"name": name, **c} if name else c


def _rope(name, inverse, seqs, toks, heads, d_head, axes, t, pairing="interleaved", joint=False, far=0, packed=True):
    # axes: widths of the rotated parts of a head, one per position axis; far: added to the first axis' positions;
    # packed: q and k are views into [seqs, toks, 3, heads, d_head], else a tensor of their own
    c = {"op": "rope", "inverse": inverse, "seqs": seqs, "toks": toks, "heads": heads, "d_head": d_head,
         "axes": ",".join(str(a) for a in axes), "t": t, "pairing": pairing, "joint": joint, "far": far, "packed": packed}
    return {"name": name, **c} if name else c


def _gated(name, back, M, F, K, t, act="silu", bias=True):
    c = {"op": "gated_bwd" if back else "gated", "M": M, "F": F, "K": K, "t": t, "act": act, "bias": bias}
    return {"name": name, **c} if name else c


def listed():
    return [
        # adaptive norm of one 256-token sequence of a small model (width 384): a launch more than a transfer
        _norm("norm_small", False, 1, 256, 384, "fp32", "bf16"),
        # the norm in front of a block's linear layers: 24 sequences of 1024 tokens, width 1152, fp32 residual stream
        _norm("norm_xl", False, 24, 1024, 1152, "fp32", "bf16"),
        # its backward pass, with the gradient of the residual path added and the modulation's gradient per sequence
        _norm("norm_bwd_xl", True, 24, 1024, 1152, "fp32", "bf16"),
        # a norm with a learned weight over a ragged number of rows of an odd width, everything bf16
        _norm("norm_bwd_odd", True, 1, 5003, 1001, "bf16", "bf16", "plain"),
        # queries and keys of 24 images of 32 x 32 patches inside the packed projection (16 heads of 72: 36 + 36)
        _rope("rope_image", False, 24, 1024, 16, 72, (36, 36), "bf16"),
        # a clip of 16 frames (time, height, width), its gradient on the way back, fp32
        _rope("rope_clip_inverse", True, 2, 4096, 16, 72, (24, 24, 24), "fp32", pairing="halves", joint=True, far=100000),
        # one image of a small model, 6 heads of 64
        _rope("rope_small", False, 1, 256, 6, 64, (32, 32), "bf16"),
        # one token through the feed-forward layer of a width-1152 model: the weights' bytes are the time
        _gated("gated_token", False, 1, 4608, 1152, "bf16"),
        # the feed-forward layer over 24 sequences of 1024 tokens, pre-activations kept for the backward pass
        _gated("gated_xl", False, 24 * 1024, 4608, 1152, "bf16"),
        # the exact mode on a small model's widths, a ragged number of rows
        _gated("gated_fp32", False, 1030, 1536, 384, "fp32", "gelu"),
        # gradients of the same layer: of the input, of both weight halves and of the bias
        _gated("gated_bwd_xl", True, 24 * 1024, 4608, 1152, "bf16"),
        # gradients for a small model and a ragged batch: few tiles, a long sum over rows
        _gated("gated_bwd_small", True, 4 * 1024 + 77, 1536, 384, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_bwd", "rope", "rope", "gated", "gated_bwd"])
    if kind in ("norm", "norm_bwd"):
        D = _log(rng, 40, 4600)
        if rng.random() < 0.7:
            D = max(8, D // 8 * 8)
        weight = rng.choice(["unit", "unit", "plain", "none"])
        groups = 1 if weight != "unit" else _log(rng, 1, 64)
        rows = _log(rng, 1, max(1, min(32768, 24 * 1024 * 1152 // (D * groups))))
        return _norm(None, kind == "norm_bwd", groups, rows, D, rng.choice(["fp32", "bf16"]), rng.choice(["bf16", "fp32"]), weight)
    if kind == "rope":
        heads, d_head = rng.choice([1, 2, 6, 12, 16, 24]), rng.choice([16, 32, 64, 72, 80, 96, 128])
        n = rng.choice([1, 2, 3])
        axes = [2 * max(1, d_head // 2 // n) for _ in range(n)]
        if rng.random() < 0.3:                                   # part of the head is left as it is
            axes[-1] = max(2, axes[-1] // 4 * 2)
        toks = _log(rng, 1, 8192)
        seqs = _log(rng, 1, max(1, min(32, 24 * 1024 * 16 * 72 // (toks * heads * d_head))))
        return _rope(None, rng.random() < 0.4, seqs, toks, heads, d_head, axes, rng.choice(["bf16", "bf16", "fp32"]),
                     rng.choice(["interleaved", "halves"]), rng.random() < 0.4, rng.choice([0, 0, 1000, 300000]), rng.random() < 0.5)
    t = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    K, F = _log(rng, 64, 2048), _log(rng, 128, 6000)
    if t == "bf16":
        K, F = K // 8 * 8, F // 8 * 8
    most = (24 * 1024 * 4608 * 1152) if t == "bf16" else (4096 * 1536 * 384)
    M = _log(rng, 1, max(1, min(32768, most // (F * K))))
    return _gated(None, kind == "gated_bwd", M, F, K, t, rng.choice(["silu", "gelu"]), rng.random() < 0.7)


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _positions(case):
    """Patch positions of a token sequence on its axes: a (time,) height, width grid as near to a square as it gets."""
    n, toks = len(case["axes"].split(",")), case["toks"]
    i = torch.arange(toks, device="cuda", dtype=torch.int64)
    if n == 1:
        p = [i]
    else:
        side = max(1, math.isqrt(toks)) if n == 2 else max(1, round(toks ** (1.0 / 3.0)))
        p = [i // side, i % side] if n == 2 else [i // (side * side), i // side % side, i % side]
    p[0] = p[0] + case["far"]
    return torch.stack(p, dim=1).to(torch.float32)


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    if op in ("norm", "norm_bwd"):
        n, r, D = case["groups"], case["rows"], case["D"]
        # a residual stream: unit noise plus an offset per channel and a scale per row
        x = (_randn(g, n * r, D) * (0.5 + torch.rand(n * r, 1, generator=g, device="cuda")) + 0.5 * _randn(g, 1, D)).to(_T[case["x"]])
        w = b = None
        if case["weight"] != "none":
            w, b = 0.2 * _randn(g, n, D), 0.2 * _randn(g, n, D)
            if case["weight"] == "plain":
                w = w + 1
        st = {"x": x, "w": w, "b": b, "case": case}
        if op == "norm_bwd":
            # what the forward pass kept, and the gradients that arrive
            xd = x.double()
            mu = xd.mean(1)
            rstd = (xd.var(1, unbiased=False) + 1e-6).rsqrt()
            st["stats"] = torch.stack([mu, rstd], dim=1).float()
            st["dy"] = (0.1 * _randn(g, n * r, D)).to(_T[case["y"]])
            st["dres"] = (0.1 * _randn(g, n * r, D)).to(_T[case["x"]])
        return st
    if op == "rope":
        s, t, h, d = case["seqs"], case["toks"], case["heads"], case["d_head"]
        if case["packed"]:                                        # q and k heads inside the packed projection
            x = _randn(g, s, t, 3 * h, d).to(_T[case["t"]])[:, :, :2 * h]
        else:
            x = _randn(g, s, t, h, d).to(_T[case["t"]])
        return {"x": x, "pos": _positions(case), "axes": tuple(int(a) for a in case["axes"].split(",")), "case": case}
    M, F, K, t = case["M"], case["F"], case["K"], _T[case["t"]]
    st = {"x": _randn(g, M, K).to(t), "w": (_randn(g, 2 * F, K) / math.sqrt(K)).to(t),
          "b": 0.1 * _randn(g, 2 * F) if case["bias"] else None, "case": case}
    if op == "gated_bwd":
        st["pre"] = _randn(g, M, 2 * F).to(t)
        st["dh"] = (0.05 * _randn(g, M, F)).to(t)
    return st


# ------------------------------------------------------------------------------------------------ plain forms
def _rows(v, n, r):
    """[n, D] per group -> [n * r, D] per row (a view where there is one group)."""
    return v.unsqueeze(1).expand(v.shape[0], r, v.shape[1]).reshape(n * r, v.shape[1])


def _plain_norm(s):
    c = s["case"]
    x = s["x"].float()
    mu = x.mean(1, keepdim=True)
    d = x - mu
    rstd = (d.square().mean(1, keepdim=True) + 1e-6).rsqrt()
    y = d * rstd
    if s["w"] is not None:
        w = s["w"] + 1 if c["weight"] == "unit" else s["w"]
        y = y * _rows(w, c["groups"], c["rows"]) + _rows(s["b"], c["groups"], c["rows"])
    return {"y": y.to(_T[c["y"]]), "stats": torch.cat([mu, rstd], dim=1)}


def _plain_norm_bwd(s):
    c = s["case"]
    n, r, D = c["groups"], c["rows"], c["D"]
    dy, rstd = s["dy"].float(), s["stats"][:, 1:]
    xhat = (s["x"].float() - s["stats"][:, :1]) * rstd
    g = dy
    out = {}
    if s["w"] is not None:
        w = s["w"] + 1 if c["weight"] == "unit" else s["w"]
        g = dy * _rows(w, n, r)
        out["dw"] = (dy * xhat).view(n, r, D).sum(1)
        out["db"] = dy.view(n, r, D).sum(1)
    dx = (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True)) * rstd + s["dres"].float()
    return {"dx": dx.to(_T[c["x"]]), **out}


def _frequencies(axes, joint, dtype, device):
    """Angle per unit of position and the axis, for every rotated pair."""
    parts, which, total = [], [], sum(axes)
    at = 0
    for a, w in enumerate(axes):
        i = torch.arange(w // 2, dtype=dtype, device=device)
        parts.append(10000.0 ** (-2.0 * (i + at) / total) if joint else 10000.0 ** (-2.0 * i / w))
        which.append(torch.full((w // 2,), a, dtype=torch.int64, device=device))
        at += w // 2
    return torch.cat(parts), torch.cat(which)


def _plain_rope(s):
    c, x = s["case"], s["x"]
    total = sum(s["axes"])
    freq, axis = _frequencies(s["axes"], c["joint"], torch.float64, x.device)
    ang = s["pos"].double()[:, axis] * freq                       # [toks, pairs]
    if c["inverse"]:
        ang = -ang
    cos, sin = ang.cos().float()[None, :, None], ang.sin().float()[None, :, None]
    v = x[..., :total].float()
    if c["pairing"] == "interleaved":
        a, b = v[..., 0::2], v[..., 1::2]
        rot = torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)
    else:
        a, b = v[..., :total // 2], v[..., total // 2:]
        rot = torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
    return torch.cat([rot.to(x.dtype), x[..., total:]], dim=-1)


_GELU_A, _GELU_B = math.sqrt(2.0 / math.pi), 0.044715


def _act(kind, g):
    """The activation and its derivative."""
    if kind == "silu":
        s = 1 / (1 + (-g).exp())
        return g * s, s * (1 + g * (1 - s))
    t = (_GELU_A * (g + _GELU_B * g * g * g)).tanh()
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * _GELU_A * (1 + 3 * _GELU_B * g * g)


def _plain_gated(s):
    c = s["case"]
    z = s["x"].float() @ s["w"].float().t()
    if s["b"] is not None:
        z = z + s["b"]
    h = _act(c["act"], z[:, :c["F"]])[0] * z[:, c["F"]:]
    return {"h": h.to(s["x"].dtype), "pre": z.to(s["x"].dtype)}


def _plain_gated_bwd(s):
    c, t = s["case"], s["x"].dtype
    F = c["F"]
    dh, g, u = s["dh"].float(), s["pre"][:, :F].float(), s["pre"][:, F:].float()
    a, da = _act(c["act"], g)
    dz = torch.cat([dh * u * da, dh * a], dim=1)
    out = {"dx": (dz @ s["w"].float()).to(t), "dw": (dz.t() @ s["x"].float()).to(t)}
    if s["b"] is not None:
        out["db"] = dz.sum(0)
    return out


_PLAIN = {"norm": _plain_norm, "norm_bwd": _plain_norm_bwd, "rope": _plain_rope, "gated": _plain_gated, "gated_bwd": _plain_gated_bwd}


# ------------------------------------------------------------------------------------------------ the framework's calls
def _own(s):
    import paper_2511_20390_b200 as free
    c = s["case"]
    op = c["op"]
    if op == "norm":
        y, stats = free.op_layer_norm(s["x"], s["w"], s["b"], rows_per_group=c["rows"], unit_offset=c["weight"] == "unit", eps=1e-6,
                                      out_dtype=_T[c["y"]], want_stats=True)
        return {"y": y, "stats": stats}
    if op == "norm_bwd":
        dx, dw, db = free.op_layer_norm_bwd(s["x"], s["dy"], s["stats"], s["w"], rows_per_group=c["rows"],
                                            unit_offset=c["weight"] == "unit", dres=s["dres"])
        return {"dx": dx} if s["w"] is None else {"dx": dx, "dw": dw, "db": db}
    if op == "rope":
        return free.op_rope_axes(s["x"], s["pos"], s["axes"], base=10000.0, pairing=c["pairing"], joint_freq=c["joint"], inverse=c["inverse"])
    if op == "gated":
        h, pre = free.op_gated_linear(s["x"], s["w"], s["b"], act=c["act"], want_preact=True)
        return {"h": h, "pre": pre}
    dx, dw, db = free.op_gated_linear_bwd(s["x"], s["w"], s["pre"], s["dh"], act=c["act"], want_dbias=c["bias"])
    return {"dx": dx, "dw": dw, "db": db} if c["bias"] else {"dx": dx, "dw": dw}


def run(state):
    if own:
        return _own(state)
    return _PLAIN[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------ work
def work(case):
    op = case["op"]
    if op in ("norm", "norm_bwd"):
        n, r, D = case["groups"], case["rows"], case["D"]
        e, bx, by = n * r * D, _BYTES[case["x"]], _BYTES[case["y"]]
        vec = 0 if case["weight"] == "none" else n * D * 4
        if op == "norm":
            return {"bytes": e * (bx + by) + 2 * vec + n * r * 8, "flops": 8 * e}
        return {"bytes": e * (3 * bx + by) + 3 * vec + n * r * 8, "flops": 16 * e}
    if op == "rope":
        e = case["seqs"] * case["toks"] * case["heads"] * (2 if case["packed"] else 1) * case["d_head"]
        return {"bytes": 2 * e * _BYTES[case["t"]] + case["toks"] * len(case["axes"].split(",")) * 4, "flops": 3 * e}
    M, F, K, b = case["M"], case["F"], case["K"], _BYTES[case["t"]]
    if op == "gated":
        return {"bytes": b * (M * K + 2 * F * K + 3 * M * F) + (8 * F if case["bias"] else 0), "flops": 4 * M * F * K}
    return {"bytes": b * (2 * M * K + 4 * F * K + 3 * M * F) + (8 * F if case["bias"] else 0), "flops": 8 * M * F * K}


# ------------------------------------------------------------------------------------------------ 64 bits
def _exact_norm(case, s):
    n, r, D = case["groups"], case["rows"], case["D"]
    x = s["x"].double().view(n, r, D)
    var, mu = torch.var_mean(x, dim=2, correction=0, keepdim=True)
    inv = 1.0 / torch.sqrt(var + 1e-6)
    xh = (x - mu) * inv
    gain = None
    if s["w"] is not None:
        gain = (s["w"].double() + (1.0 if case["weight"] == "unit" else 0.0)).view(n, 1, D)
    if case["op"] == "norm":
        y = xh if gain is None else torch.addcmul(s["b"].double().view(n, 1, D), xh, gain)
        return {"y": y.reshape(n * r, D), "stats": torch.stack([mu.reshape(-1), inv.reshape(-1)], dim=1)}
    # the kept statistics are inputs of the backward pass
    mu, inv = s["stats"][:, 0].double().view(n, r, 1), s["stats"][:, 1].double().view(n, r, 1)
    xh = (x - mu) * inv
    dy = s["dy"].double().view(n, r, D)
    v = dy if gain is None else dy * gain
    proj = torch.einsum("nrd,nrd->nr", v, xh).unsqueeze(2) / D
    dx = s["dres"].double().view(n, r, D) + inv * (v - v.sum(2, keepdim=True) / D - proj * xh)
    out = {"dx": dx.reshape(n * r, D)}
    if gain is not None:
        out["dw"], out["db"] = torch.einsum("nrd,nrd->nd", dy, xh), dy.sum(1)
    return out


def _exact_rope(case, s):
    x = s["x"].double()
    axes, total = s["axes"], sum(s["axes"])
    turns = []
    first = 0
    for a, width in enumerate(axes):
        for i in range(width // 2):
            e = (first + i) / (total / 2) if case["joint"] else i / (width / 2)
            turns.append(s["pos"][:, a].double() * math.exp(-e * math.log(10000.0)))
        first += width // 2
    ang = torch.stack(turns, dim=1)
    z = torch.polar(torch.ones_like(ang), -ang if case["inverse"] else ang)[None, :, None, :]
    out = x.clone()
    if case["pairing"] == "interleaved":
        out[..., :total] = torch.view_as_real(torch.view_as_complex(x[..., :total].unflatten(-1, (total // 2, 2)).contiguous()) * z).flatten(-2)
    else:
        w = torch.complex(x[..., :total // 2], x[..., total // 2:total]) * z
        out[..., :total // 2], out[..., total // 2:total] = w.real, w.imag
    return out


def _exact_gated(case, s):
    F = case["F"]
    w = s["w"].double()
    if case["op"] == "gated":
        z = torch.nn.functional.linear(s["x"].double(), w, None if s["b"] is None else s["b"].double())
    else:
        z = s["pre"].double()
    g, u = z[:, :F], z[:, F:]
    if case["act"] == "silu":
        sg = torch.special.expit(g)
        a, slope = g * sg, sg + g * sg * torch.special.expit(-g)
    else:                                                          # tanh form: (1 + tanh v) / 2 is the logistic function of 2 v
        sg = torch.special.expit(2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3))
        a = g * sg
        slope = sg + g * sg * (1 - sg) * 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * g ** 2)
    if case["op"] == "gated":
        return {"h": a * u, "pre": z}
    dh = s["dh"].double()
    dg, du = dh * u * slope, dh * a
    x = s["x"].double()
    out = {"dx": dg @ w[:F] + du @ w[F:], "dw": torch.cat([dg.t() @ x, du.t() @ x])}
    if s["b"] is not None:
        out["db"] = torch.cat([dg.sum(0), du.sum(0)])
    return out


def exact(case, seed):
    s = prepare(case, seed)
    with torch.no_grad():
        if case["op"] in ("norm", "norm_bwd"):
            return _exact_norm(case, s)
        if case["op"] == "rope":
            return _exact_rope(case, s)
        return _exact_gated(case, s)
