"""Operators of text-conditioned transformer blocks as cases to measure: attention of a sequence's tokens to an encoder's
states of another length and its backward pass, and the root-mean-square norm with the residual's addition (16-, 32- or
8-bit results) and its backward pass.

`run` computes a case either in its plain form, with elementary torch operations in 32 bits, or (where `own` is true)
with this framework's operators; `exact` gives the same outputs from the definitions in 64 bits.
"""
import math

import torch

own = False

_T = {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}
_BYTES = {"bf16": 2, "fp32": 4, "e4m3": 1, "none": 0}


# ------------------------------------------------------------------------------------------------ cases
def _cross(name, back, seqs, enc, n_q, n_kv, heads, kv_heads, d, t, lens="ragged", layout="padded", mask=False):
    # seqs sequences of n_q tokens read enc encoder sequences of up to n_kv states (seqs / enc consecutive ones share one);
    # lens: "full", "ragged", or "empty" (ragged, and every third encoder sequence has no state at all);
    # layout: "padded" [enc, n_kv, ...] or "packed" (the states of all sequences one behind the other); mask: holes in the states
    c = {"op": "cross_bwd" if back else "cross", "seqs": seqs, "enc": enc, "n_q": n_q, "n_kv": n_kv, "heads": heads,
         "kv_heads": kv_heads, "d": d, "t": t, "lens": lens, "layout": layout, "mask": mask}
    return {"name": name, **c} if name else c


def _rms(name, back, rows, heads, D, x, res, y, weight="plain", block=0, groups=1):
    # heads > 0: a norm over every head of D elements inside a packed projection [rows, 3, heads, D], else over rows of D;
    # res: type of the residual stream or "none"; weight: "unit" = 1 + scale per group of rows, "plain" = a learned weight, "none";
    # block: columns that share a scale of an 8-bit result (0: the row)
    c = {"op": "rms_bwd" if back else "rms", "rows": rows, "heads": heads, "D": D, "x": x, "res": res, "y": y, "weight": weight,
         "block": block, "groups": groups}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one pooled token per image over a short prompt: a launch more than a transfer
        _cross("cross_token", False, 4, 4, 1, 77, 6, 6, 64, "bf16"),
        # single tokens over long encoders, shared key heads: the cache's bytes are the time
        _cross("cross_token_long", False, 8, 8, 1, 16384, 32, 8, 128, "bf16"),
        # the packed pass of four images, six drafts each, 1024 tokens, 16 heads of 72: the drafts of an image share its prompt
        _cross("cross_drafts", False, 24, 4, 1024, 300, 16, 16, 72, "bf16"),
        # long sequences of a wide model over long prompts, encoder states packed
        _cross("cross_large", False, 8, 8, 4096, 512, 16, 16, 128, "bf16", "ragged", "packed"),
        # the exact mode on a small model: odd lengths, holes in the states, an encoder sequence without any
        _cross("cross_fp32", False, 3, 3, 333, 77, 6, 6, 40, "fp32", "empty", "padded", True),
        # gradients of the training step of 24 images with a prompt each
        _cross("cross_bwd_xl", True, 24, 24, 1024, 300, 16, 16, 72, "bf16"),
        # gradients on a small model, short prompts packed, two query heads to a key head
        _cross("cross_bwd_small", True, 4, 4, 256, 120, 6, 3, 64, "bf16", "empty", "packed"),
        # the norm of one 256-token sequence of a small model (width 384)
        _rms("rms_small", False, 256, 0, 384, "bf16", "none", "bf16"),
        # a block's addition to the fp32 residual stream and the modulated norm behind it, 24 sequences of 1024 tokens
        _rms("rms_residual", False, 24 * 1024, 0, 1152, "bf16", "fp32", "bf16", "unit", 0, 24),
        # the norm of all queries' heads inside the packed projection
        _rms("rms_heads", False, 24 * 1024, 16, 72, "bf16", "none", "bf16"),
        # residual addition, norm and an 8-bit operand with a scale per 128 columns for the product behind it
        _rms("rms_8bit", False, 4100, 0, 4096, "bf16", "bf16", "e4m3", "plain", 128),
        # the backward pass of the second, with the gradient that reaches the stream past the norm
        _rms("rms_bwd", True, 24 * 1024, 0, 1152, "fp32", "fp32", "bf16", "unit", 0, 24),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    if rng.random() < 0.6:
        back = rng.random() < 0.4
        t = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        d = rng.choice([32, 40, 64, 72, 80, 96, 128])
        heads = rng.choice([1, 2, 4, 6, 8, 12, 16])
        kv_heads = rng.choice([h for h in (1, 2, 3, 4, 6, 8, 12, 16) if heads % h == 0 and h * 8 >= heads] + [heads] * 3)
        n_q = 1 if not back and rng.random() < 0.3 else _log(rng, 2, 4096)
        n_kv = _log(rng, 1, 16384 if n_q == 1 else 2048)
        most = 24 * 1024 * 300 * 16 * 72 if back else 8 * 4096 * 512 * 16 * 128
        if t == "fp32":
            most //= 40
        most = min(most, (24 * 1024 * 16 * 72 if back else 8 * 4096 * 16 * 128) * n_kv)
        while n_q * n_kv * heads * d > most:
            n_q, n_kv = max(1, n_q // 2), max(1, n_kv * 2 // 3)
        enc = _log(rng, 1, max(1, min(24, most // (n_q * n_kv * heads * d))))
        share = rng.choice([s for s in (1, 1, 2, 3, 6) if s == 1 or enc * s * n_q * n_kv * heads * d <= most])
        return _cross(None, back, enc * share, enc, n_q, n_kv, heads, kv_heads, d, t, rng.choice(["full", "ragged", "ragged", "empty"]),
                      rng.choice(["padded", "padded", "packed"]), rng.random() < 0.2)
    back = rng.random() < 0.4
    heads = rng.choice([0, 0, 0, 1, 6, 12, 16])
    D = rng.choice([32, 40, 64, 72, 80, 96, 128]) if heads else _log(rng, 40, 8000)
    if D > 128 and rng.random() < 0.75:
        D = D // 8 * 8
    x = rng.choice(["bf16", "bf16", "fp32"])
    res = "none" if heads else rng.choice(["none", "bf16", "fp32"])
    y = rng.choice(["bf16", "fp32"]) if back or heads else rng.choice(["bf16", "bf16", "fp32", "e4m3", "e4m3"])
    rows = _log(rng, 1, min(32768, 24 * 1024 * 1152 // (D * max(heads, 1))))
    weight = rng.choice(["plain", "plain", "unit", "none"])
    groups = 1
    if weight == "unit" and not heads:
        groups = _log(rng, 1, 24)
        rows = max(1, rows // groups) * groups
    if back:
        x = res if res != "none" else x
    return _rms(None, back, rows, heads, D, x, res, y, weight, rng.choice([0, 128]) if y == "e4m3" else 0, groups)


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _lens(c):
    """States of every encoder sequence."""
    out = []
    for e in range(c["enc"]):
        n = c["n_kv"] if c["lens"] == "full" else max(1, c["n_kv"] - int(0.8 * c["n_kv"] * (e * 0.6180339887 % 1.0)))
        out.append(0 if c["lens"] == "empty" and e % 3 == 1 else n)
    return out


def _prepare_cross(c, g):
    s, e, n, m, h, kh, d, t = (c[k] for k in ("seqs", "enc", "n_q", "n_kv", "heads", "kv_heads", "d", "t"))
    lens = _lens(c)
    packed = c["layout"] == "packed"
    q = _randn(g, s, n, h, d).to(_T[t])
    # keys and values side by side, as one projection of the encoder's states leaves them
    lead = (max(1, sum(lens)),) if packed else (e, m)
    kv = _randn(g, *lead, 2, kh, d).to(_T[t])
    st = {"q": q, "k": kv[..., 0, :, :], "v": kv[..., 1, :, :], "case": c, "mask": None}
    at = [0]
    for x in lens:
        at.append(at[-1] + x)
    st["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    st["offsets"] = torch.tensor(at, dtype=torch.int32, device="cuda")
    st["longest"] = max(lens)
    if c["mask"]:
        st["mask"] = torch.rand(*lead, generator=g, device="cuda") < 0.9
    if c["op"] == "cross_bwd":
        st["out"], st["lse"] = _plain_cross(st).values()           # what the forward pass kept, and the gradient that arrives
        st["dout"] = (0.1 * _randn(g, s, n, h, d)).to(_T[t])
    return st


def _prepare_rms(c, g):
    rows, h, D, n = c["rows"], c["heads"], c["D"], c["groups"]
    scale = 0.5 + torch.rand(rows, 1, generator=g, device="cuda")
    if h:
        x = _randn(g, rows, 3, h, D).to(_T[c["x"]])[:, 0]
    else:
        x = (_randn(g, rows, D) * scale).to(_T[c["x"]])
    st = {"x": x, "res": None, "w": None, "case": c}
    if c["weight"] != "none":
        st["w"] = 0.2 * _randn(g, n, D) + (1.0 if c["weight"] == "plain" else 0.0)
    if c["op"] == "rms":
        if c["res"] != "none":
            st["res"] = (2.0 * scale * _randn(g, rows, D)).to(_T[c["res"]])
        return st
    # what the forward pass kept, and the gradients that arrive: at the result, and at the residual stream behind the addition
    st["rstd"] = (x.double().square().mean(-1) + 1e-6).rsqrt().float().reshape(-1)
    shape = (rows, h, D) if h else (rows, D)
    st["dy"] = (0.1 * _randn(g, *shape)).to(_T[c["y"]])
    if c["res"] != "none":
        st["dres"] = (0.1 * _randn(g, *shape)).to(_T[c["x"]])
    return st


def prepare(case, seed):
    g = _gen(seed)
    return _prepare_cross(case, g) if case["op"].startswith("cross") else _prepare_rms(case, g)


# ------------------------------------------------------------------------------------------------ plain forms
def _states(s, x):
    """Encoder states as [enc, n, kv_heads, d] in 32 bits (zeros where there is none) and which of them count."""
    c = s["case"]
    n = max(1, s["longest"])
    i = torch.arange(n, device=x.device)
    valid = i[None, :] < s["lens"][:, None]
    if c["layout"] == "packed":
        at = (s["offsets"][:-1, None] + i[None, :]).clamp(max=x.shape[0] - 1).long()
        x, mask = x[at], None if s["mask"] is None else s["mask"][at]
    else:
        x, mask = x[:, :n], None if s["mask"] is None else s["mask"][:, :n]
    if mask is not None:
        valid = valid & mask
    return torch.where(valid[:, :, None, None], x.float(), 0.0), valid


def _per_seq(c, x):
    """[enc, n, kv_heads, d] -> [seqs, heads, n, d]: every sequence's and every query head's own."""
    x = x.repeat_interleave(c["seqs"] // c["enc"], 0).repeat_interleave(c["heads"] // c["kv_heads"], 2)
    return x.permute(0, 2, 1, 3)


def _probabilities(s, k, valid):
    c = s["case"]
    q = s["q"].float().permute(0, 2, 1, 3) * (1.0 / math.sqrt(c["d"]))
    score = q @ _per_seq(c, k).transpose(2, 3)
    live = valid.repeat_interleave(c["seqs"] // c["enc"], 0)[:, None, None, :]
    return score.masked_fill_(~live, float("-inf")), live


def _plain_cross(s):
    c = s["case"]
    k, valid = _states(s, s["k"])
    v, _ = _states(s, s["v"])
    score, _ = _probabilities(s, k, valid)
    top = score.amax(3, keepdim=True)
    top = torch.where(top == float("-inf"), 0.0, top)              # rows without any state
    p = (score - top).exp_()
    total = p.sum(3, keepdim=True)
    o = (p @ _per_seq(c, v)) / torch.where(total == 0, 1.0, total)
    return {"out": o.permute(0, 2, 1, 3).contiguous().to(s["q"].dtype), "lse": (top + total.log())[..., 0]}


def _to_heads(c, x):
    """Gradients [seqs, heads, n, d] summed over the sequences and query heads that share a state: [enc, n, kv_heads, d]."""
    sh, gr = c["seqs"] // c["enc"], c["heads"] // c["kv_heads"]
    return x.reshape(c["enc"], sh, c["kv_heads"], gr, x.shape[2], x.shape[3]).sum((1, 3)).permute(0, 2, 1, 3)


def _to_layout(s, x):
    """[enc, n, kv_heads, d] in the layout and type of the states, zeros where there is none."""
    c = s["case"]
    out = torch.zeros(s["k"].shape, dtype=s["k"].dtype, device=x.device)
    if c["layout"] == "packed":
        i = torch.arange(x.shape[1], device=x.device)
        live = i[None, :] < s["lens"][:, None]
        out[(s["offsets"][:-1, None] + i[None, :])[live].long()] = x[live].to(out.dtype)
    else:
        out[:, :x.shape[1]] = x.to(out.dtype)
    return out


def _plain_cross_bwd(s):
    c = s["case"]
    k, valid = _states(s, s["k"])
    v, _ = _states(s, s["v"])
    score, live = _probabilities(s, k, valid)
    p = torch.where(live, (score - s["lse"][..., None]).exp_(), 0.0)
    del score
    do, o = s["dout"].float().permute(0, 2, 1, 3), s["out"].float().permute(0, 2, 1, 3)
    dv = _to_heads(c, p.transpose(2, 3) @ do)
    dp = do @ _per_seq(c, v).transpose(2, 3)
    ds = p.mul_(dp.sub_((do * o).sum(3, keepdim=True))).mul_(1.0 / math.sqrt(c["d"]))
    dq = ds @ _per_seq(c, k)
    dk = _to_heads(c, ds.transpose(2, 3) @ s["q"].float().permute(0, 2, 1, 3))
    return {"dq": dq.permute(0, 2, 1, 3).contiguous().to(s["q"].dtype), "dk": _to_layout(s, dk), "dv": _to_layout(s, dv)}


def _weights(s):
    """The weight of every row, [rows, D] or [D], or 1."""
    c = s["case"]
    if s["w"] is None:
        return 1.0
    w = s["w"] + 1 if c["weight"] == "unit" else s["w"]
    if c["groups"] == 1:
        return w[0]
    return w.unsqueeze(1).expand(-1, c["rows"] // c["groups"], -1).reshape(c["rows"], c["D"])


def _blocks(y, block):
    """[rows, D] -> [rows, blocks, columns of a block], the last one filled up with zeros."""
    n = y.shape[1] if block == 0 else block
    pad = -y.shape[1] % n
    if pad:
        y = torch.cat([y, y.new_zeros(y.shape[0], pad)], dim=1)
    return y.view(y.shape[0], -1, n)


def _values(q, scales, D):
    """What 8-bit results and their scales stand for, in the model's 16 bits."""
    v = q.to(torch.bfloat16)                                       # every 8-bit number is a 16-bit one; products are rounded once
    blocks = scales.shape[1]
    if blocks == 1 or D % 128 == 0:
        return v.view(-1, blocks, D // blocks).mul_(scales[:, :, None]).view(-1, D)
    return v.mul_(scales.repeat_interleave(128, 1)[:, :D])


def _plain_rms(s):
    c = s["case"]
    h = s["x"].float()
    out = {}
    if s["res"] is not None:
        h = h + s["res"].float()
        out["h"] = h.to(s["res"].dtype)
    rstd = (h.square().mean(-1, keepdim=True) + 1e-6).rsqrt()
    y = h * rstd * _weights(s)
    if c["y"] == "e4m3":
        b = _blocks(y, c["block"])
        top = b.abs().amax(2)
        scales = torch.where(top < 2.0 ** -100, 1.0, top / 448.0)
        q = (b / scales[:, :, None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
        out["y"] = _values(q.reshape(y.shape[0], -1)[:, :c["D"]], scales, c["D"])
        out["scales"] = scales
    else:
        out["y"] = y.to(_T[c["y"]])
    out["rstd"] = rstd.reshape(-1)
    return out


def _plain_rms_bwd(s):
    c = s["case"]
    h, dy = s["x"].float(), s["dy"].float()
    rstd = s["rstd"].view(*h.shape[:-1], 1)
    xh = h * rstd
    v = dy * _weights(s)
    dx = (v - xh * (v * xh).mean(-1, keepdim=True)) * rstd
    if c["res"] != "none":
        dx = dx + s["dres"].float()
    out = {"dx": dx.to(s["x"].dtype)}
    if s["w"] is not None:
        out["dw"] = (dy * xh).reshape(c["groups"], -1, c["D"]).sum(1)
    return out


_PLAIN = {"cross": _plain_cross, "cross_bwd": _plain_cross_bwd, "rms": _plain_rms, "rms_bwd": _plain_rms_bwd}


# ------------------------------------------------------------------------------------------------ the framework's calls
def _own(s):
    import paper_2511_20390_b200 as free
    c = s["case"]
    op = c["op"]
    if op.startswith("cross"):
        where = {"kv_offsets": s["offsets"], "max_kv": c["n_kv"]} if c["layout"] == "packed" else {"kv_lens": s["lens"]}
        if op == "cross":
            out, lse = free.op_cross_attention(s["q"], s["k"], s["v"], kv_mask=s["mask"], want_lse=True, **where)
            return {"out": out, "lse": lse}
        dq, dk, dv = free.op_cross_attention_bwd(s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"], kv_mask=s["mask"], **where)
        return {"dq": dq, "dk": dk, "dv": dv}
    h = c["heads"]
    form = {"rows_per_group": c["rows"] * max(h, 1) // c["groups"], "unit_offset": c["weight"] == "unit"}
    if op == "rms_bwd":
        dx, dw = free.op_rms_norm_bwd(s["x"], s["dy"], s["rstd"], s["w"], dres=s.get("dres"), want_dweight=s["w"] is not None, **form)
        return {"dx": dx} if dw is None else {"dx": dx, "dw": dw}
    r = free.op_rms_norm(s["x"], s["w"], residual=s["res"], eps=1e-6, out_dtype=_T[c["y"]], scale_block=c["block"] or None,
                         want_rstd=True, **form)
    out = {} if s["res"] is None else {"h": r.residual}
    if c["y"] == "e4m3":
        out["y"], out["scales"] = _values(r.y, r.scales, c["D"]), r.scales
    else:
        out["y"] = r.y
    out["rstd"] = r.rstd
    return out


def run(state):
    if own:
        return _own(state)
    return _PLAIN[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------ work
def work(case):
    c = case
    if c["op"].startswith("cross"):
        lens, b = _lens(c), _BYTES[c["t"]]
        share = c["seqs"] // c["enc"]
        qe, ke = c["seqs"] * c["n_q"] * c["heads"] * c["d"], sum(lens) * c["kv_heads"] * c["d"]
        stats = 4 * c["seqs"] * c["n_q"] * c["heads"]
        pairs = share * sum(lens) * c["n_q"] * c["heads"] * c["d"]
        if c["op"] == "cross":
            return {"bytes": b * (2 * qe + 2 * ke) + stats, "flops": 4 * pairs}
        return {"bytes": b * (4 * qe + 4 * ke) + stats, "flops": 10 * pairs}
    e = c["rows"] * max(c["heads"], 1) * c["D"]
    vec = 0 if c["weight"] == "none" else 4 * c["groups"] * c["D"]
    stats = 4 * c["rows"] * max(c["heads"], 1)
    if c["op"] == "rms":
        scales = 0 if c["y"] != "e4m3" else 4 * c["rows"] * (1 if not c["block"] else -(-c["D"] // c["block"]))
        return {"bytes": e * (_BYTES[c["x"]] + 2 * _BYTES[c["res"]] + _BYTES[c["y"]]) + vec + stats + scales, "flops": 5 * e}
    back = 3 if c["res"] != "none" else 2
    return {"bytes": e * (back * _BYTES[c["x"]] + _BYTES[c["y"]]) + 2 * vec + stats, "flops": 10 * e}


# ------------------------------------------------------------------------------------------------ 64 bits
def _exact_cross(c, s):
    """Sequence by sequence and key head by key head, only over the states that count; gradients by differentiation."""
    back = c["op"] == "cross_bwd"
    lens, at = _lens(c), [0]
    for n in lens:
        at.append(at[-1] + n)
    share, group = c["seqs"] // c["enc"], c["heads"] // c["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full((c["seqs"], c["heads"], c["n_q"]), -math.inf, dtype=torch.float64, device="cuda")
    dk, dv = (torch.zeros(s["k"].shape, dtype=torch.float64, device="cuda") for _ in range(2))
    for i in range(c["seqs"]):
        e = i // share
        span = slice(at[e], at[e + 1]) if c["layout"] == "packed" else slice(0, lens[e])
        pick = (lambda x: x[span]) if c["layout"] == "packed" else (lambda x: x[e, span])
        use = torch.arange(lens[e], device="cuda")
        if s["mask"] is not None:
            use = use[pick(s["mask"])]
        if use.numel() == 0:
            continue
        for kh in range(c["kv_heads"]):
            hs = slice(kh * group, (kh + 1) * group)
            q = s["q"][i, :, hs].double().requires_grad_(back)
            k, v = pick(s["k"])[use, kh].double().requires_grad_(back), pick(s["v"])[use, kh].double().requires_grad_(back)
            score = torch.einsum("qhd,kd->hqk", q, k) / c["d"] ** 0.5
            o = torch.einsum("hqk,kd->qhd", torch.softmax(score, dim=2), v)
            if back:
                gq, gk, gv = torch.autograd.grad(o, (q, k, v), s["dout"][i, :, hs].double())
                out[i, :, hs] = gq
                pick(dk)[use, kh] += gk
                pick(dv)[use, kh] += gv
            else:
                out[i, :, hs] = o
                lse[i, hs] = torch.logsumexp(score, dim=2)
    return {"dq": out, "dk": dk, "dv": dv} if back else {"out": out, "lse": lse}


def _round8(v):
    """To the nearest number of four bits between 2^-6 and 448 (ties to even), multiples of 2^-9 below."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(v / step) * step).clamp(-448.0, 448.0)


def _exact_rms(c, s):
    D, n = c["D"], c["groups"]
    x = s["x"].double().reshape(n, -1, D)
    gain = None if s["w"] is None else (s["w"].double() + (1.0 if c["weight"] == "unit" else 0.0)).view(n, 1, D)
    if c["op"] == "rms":
        out = {}
        if s["res"] is not None:
            x = x + s["res"].double().view_as(x)
            out["h"] = x.view(-1, D)
        size = torch.linalg.vector_norm(x, dim=2, keepdim=True)
        inv = 1.0 / torch.sqrt(size * size / D + 1e-6)
        y = x * inv if gain is None else torch.einsum("nrd,nrk,nkd->nrd", x, inv, gain)
        y = y.reshape(-1, D)
        if c["y"] == "e4m3":
            parts, scales = y.split(c["block"] or D, dim=1), []
            for i in range(len(parts)):
                top = torch.linalg.vector_norm(parts[i], ord=math.inf, dim=1, keepdim=True)
                scales.append(torch.where(top < 2.0 ** -100, torch.ones_like(top), top / 448))
            out["y"] = torch.cat([_round8(p / f) * f for p, f in zip(parts, scales)], dim=1)
            out["scales"] = torch.cat(scales, dim=1)
        else:
            out["y"] = y.reshape(s["x"].shape)
        out["rstd"] = inv.reshape(-1)
        return out
    inv = s["rstd"].double().view(n, -1, 1)                        # an input of the backward pass
    dy = s["dy"].double().reshape(n, -1, D)
    v = dy if gain is None else dy * gain
    along = torch.einsum("nrd,nrd->nr", v, x).unsqueeze(2)
    dx = inv * v - x * (inv ** 3 * along / D)
    if c["res"] != "none":
        dx = dx + s["dres"].double().view_as(dx)
    out = {"dx": dx.reshape(s["x"].shape)}
    if gain is not None:
        out["dw"] = torch.einsum("nrd,nrd,nrk->nd", dy, x, inv)
    return out


def exact(case, seed):
    c = case
    if c["op"].startswith("cross") and c["seqs"] * c["n_q"] * c["n_kv"] * c["heads"] * c["d"] * (10 if c["op"] == "cross_bwd" else 4) > 4e11:
        return None
    s = prepare(case, seed)
    return _exact_cross(c, s) if c["op"].startswith("cross") else _exact_rms(c, s)
