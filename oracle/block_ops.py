"""fp64 definitions of the transformer-block operators (numpy): layer norm with groups of rows, rotary positions with several
axes, the gated linear layer, and their backward passes.  Formulas only; shares no code with the library."""
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
