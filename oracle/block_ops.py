"""fp64 definitions of the transformer-block operators (numpy): layer norm with groups of rows, rotary positions with several
axes, the gated linear layer, the root-mean-square norm, attention to an encoder's states, and their backward passes.  Formulas only; shares no code with the library."""
import numpy as np


def _per_row(v, rows):
    return None if v is None else np.repeat(np.asarray(v, np.float64), rows, axis=0)


def layer_norm(x, weight=None, bias=None, rows_per_group=None, unit_offset=False, eps=1e-6):
    """x [M, D]; weight, bias [groups, D].  Returns (y, stats [M, 2])."""
    x = np.asarray(x, np.float64)
    rows = len(x) if rows_per_group is None else rows_per_group
    mu = x.mean(1, keepdims=True)
    r = 1.0 / np.sqrt(((x - mu) ** 2).mean(1, keepdims=True) + eps)
    y = (x - mu) * r
    if weight is not None:
        y = y * (_per_row(weight, rows) + (1.0 if unit_offset else 0.0))
    if bias is not None:
        y = y + _per_row(bias, rows)
    return y, np.concatenate([mu, r], 1)


def layer_norm_bwd(x, dy, stats, weight=None, rows_per_group=None, unit_offset=False, dres=None):
    """Returns (dx [M, D], dweight [groups, D], dbias [groups, D]) for the given mean and 1 / sqrt(var + eps) of every row."""
    x, dy, stats = (np.asarray(a, np.float64) for a in (x, dy, stats))
    M, D = x.shape
    rows = M if rows_per_group is None else rows_per_group
    xh = (x - stats[:, :1]) * stats[:, 1:]
    v = dy
    if weight is not None:
        v = dy * (_per_row(weight, rows) + (1.0 if unit_offset else 0.0))
    dx = stats[:, 1:] * (v - v.mean(1, keepdims=True) - xh * (v * xh).mean(1, keepdims=True))
    if dres is not None:
        dx = dx + np.asarray(dres, np.float64)
    g = M // rows if rows else 1
    return dx, (dy * xh).reshape(g, rows, D).sum(1), dy.reshape(g, rows, D).sum(1)


def rope_axes(x, pos, axis_dims, base=10000.0, pairing="interleaved", joint_freq=False, inverse=False):
    """x [n_seq, n_tok, heads, d_head]; pos [n_tok, n_axes] or [n_seq, n_tok, n_axes]."""
    x, pos = np.asarray(x, np.float64), np.asarray(pos, np.float64)
    if pos.ndim == 2:
        pos = np.broadcast_to(pos, (x.shape[0],) + pos.shape)
    R = sum(axis_dims)
    out = x.copy()
    p = 0
    for ax, dim in enumerate(axis_dims):
        for i in range(dim // 2):
            freq = base ** (-2.0 * p / R) if joint_freq else base ** (-2.0 * i / dim)
            t = (pos[:, :, ax] * freq)[:, :, None] * (-1.0 if inverse else 1.0)
            ia, ib = (2 * p, 2 * p + 1) if pairing == "interleaved" else (p, p + R // 2)
            a, b = x[..., ia], x[..., ib]
            out[..., ia] = a * np.cos(t) - b * np.sin(t)
            out[..., ib] = a * np.sin(t) + b * np.cos(t)
            p += 1
    return out


def gate_act(kind, g):
    """Activation of the gate and its derivative: "silu" g sigmoid(g), "gelu" the tanh form."""
    if kind == "silu":
        s = 1.0 / (1.0 + np.exp(-g))
        return g * s, s * (1.0 + g * (1.0 - s))
    k = np.sqrt(2.0 / np.pi)
    t = np.tanh(k * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * k * (1.0 + 3 * 0.044715 * g * g)


def gated_linear(x, w, bias=None, act="silu"):
    """x [M, K], w [2F, K] (gate rows, then up rows), bias [2F].  Returns (h [M, F], preact [M, 2F])."""
    z = np.asarray(x, np.float64) @ np.asarray(w, np.float64).T
    if bias is not None:
        z = z + np.asarray(bias, np.float64)
    F = z.shape[1] // 2
    return gate_act(act, z[:, :F])[0] * z[:, F:], z


def gated_linear_bwd(x, w, preact, dh, act="silu"):
    """Returns (dx [M, K], dw [2F, K], dbias [2F])."""
    x, w, z, dh = (np.asarray(a, np.float64) for a in (x, w, preact, dh))
    F = z.shape[1] // 2
    a, da = gate_act(act, z[:, :F])
    dz = np.concatenate([dh * z[:, F:] * da, dh * a], 1)
    return dz @ w, dz.T @ x, dz.sum(0)


def round_e4m3(v):
    """Nearest 8-bit number (4 bits of exponent, 3 of mantissa, up to 448), ties to the even one; NaN stays."""
    v = np.asarray(v, np.float64)
    a = np.abs(v)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.maximum(np.floor(np.log2(np.where(a > 0, a, 1.0))), -6.0)
    step = 2.0 ** (e - 3)
    return np.where(np.isnan(v), np.nan, np.copysign(np.minimum(np.round(a / step) * step, 448.0), v))


def rms_norm(x, weight=None, residual=None, rows_per_group=None, unit_offset=False, eps=1e-6):
    """x [M, D]; weight [groups, D].  Returns (y, h, r [M])."""
    h = np.asarray(x, np.float64)
    if residual is not None:
        h = h + np.asarray(residual, np.float64)
    r = 1.0 / np.sqrt((h * h).mean(1) + eps)
    y = h * r[:, None]
    if weight is not None:
        y = y * (_per_row(weight, len(h) if rows_per_group is None else rows_per_group) + (1.0 if unit_offset else 0.0))
    return y, h, r


def quantise(y, block=None):
    """8-bit values and scales [M, runs] of rows y: a run of `block` columns (None: the row) shares max |y| / 448."""
    M, D = y.shape
    n = D if block is None else block
    runs = -(-D // n)
    top = np.stack([np.abs(y[:, i * n:(i + 1) * n]).max(1) for i in range(runs)], 1)
    scales = np.where(top < 2.0 ** -100, 1.0, top / 448.0)
    return round_e4m3(y / np.repeat(scales, n, 1)[:, :D]), scales


def rms_norm_bwd(h, dy, rstd, weight=None, rows_per_group=None, unit_offset=False, dres=None):
    """Returns (dx [M, D], dweight [groups, D]) for the given 1 / sqrt(mean square + eps) of every row."""
    h, dy, r = (np.asarray(a, np.float64) for a in (h, dy, rstd))
    M, D = h.shape
    rows = M if rows_per_group is None else rows_per_group
    xh = h * r[:, None]
    v = dy if weight is None else dy * (_per_row(weight, rows) + (1.0 if unit_offset else 0.0))
    dx = r[:, None] * (v - xh * (v * xh).mean(1, keepdims=True))
    if dres is not None:
        dx = dx + np.asarray(dres, np.float64)
    return dx, (dy * xh).reshape(M // rows if rows else 1, rows, D).sum(1)


def cross_attention(q, ks, vs, counts, enc_of, scale):
    """q [n_seq, n_q, heads, d]; ks, vs: per encoder sequence [n, kv_heads, d]; counts: per encoder sequence, which states count;
    enc_of [n_seq] (out of range: none).  Returns (out like q, lse [n_seq, heads, n_q])."""
    q = np.asarray(q, np.float64)
    out, lse = np.zeros(q.shape), np.full((q.shape[0], q.shape[2], q.shape[1]), -np.inf)
    for s, e in enumerate(enc_of):
        use = np.flatnonzero(counts[e]) if 0 <= e < len(ks) else []
        if len(use) == 0:
            continue
        for h in range(q.shape[2]):
            kh = h // (q.shape[2] // ks[e].shape[1])
            S = scale * q[s, :, h] @ np.asarray(ks[e], np.float64)[use, kh].T
            top = S.max(1, keepdims=True)
            p = np.exp(S - top)
            lse[s, h] = top[:, 0] + np.log(p.sum(1))
            out[s, :, h] = (p / p.sum(1, keepdims=True)) @ np.asarray(vs[e], np.float64)[use, kh]
    return out, lse


def cross_attention_bwd(q, ks, vs, counts, enc_of, scale, out, lse, dout):
    """Gradients (dq, [dk], [dv] per encoder sequence) for the given out and lse, and for each the sum of its terms' magnitudes that a
    rounding error of every term scales with: (dq, dk, dv, mag_dq, mag_dk, mag_dv)."""
    q, out, lse, g = (np.asarray(a, np.float64) for a in (q, out, lse, dout))
    dq, mq = np.zeros(q.shape), np.zeros(q.shape)
    dk, dv, mk, mv = ([np.zeros(k.shape) for k in ks] for _ in range(4))
    for s, e in enumerate(enc_of):
        use = np.flatnonzero(counts[e]) if 0 <= e < len(ks) else []
        if len(use) == 0:
            continue
        for h in range(q.shape[2]):
            kh = h // (q.shape[2] // ks[e].shape[1])
            k, v = np.asarray(ks[e], np.float64)[use, kh], np.asarray(vs[e], np.float64)[use, kh]
            p = np.exp(scale * q[s, :, h] @ k.T - lse[s, h][:, None])
            delta = (g[s, :, h] * out[s, :, h]).sum(1, keepdims=True)
            dS = p * (g[s, :, h] @ v.T - delta) * scale
            # the bracket is a difference of sums: its error goes by the sums' terms, not by the difference
            terms = p * scale * (np.abs(g[s, :, h]) @ np.abs(v).T + np.abs(g[s, :, h] * out[s, :, h]).sum(1, keepdims=True))
            dq[s, :, h] = dS @ k
            mq[s, :, h] = terms @ np.abs(k)
            dk[e][use, kh] += dS.T @ q[s, :, h]
            mk[e][use, kh] += terms.T @ np.abs(q[s, :, h])
            dv[e][use, kh] += p.T @ g[s, :, h]
            mv[e][use, kh] += p.T @ np.abs(g[s, :, h])
    return dq, dk, dv, mq, mk, mv
