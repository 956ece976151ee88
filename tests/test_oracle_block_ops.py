"""The fp64 definitions of the block operators, pinned against torch's own functions, autograd and finite differences (CPU)."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

from oracle import block_ops as ob


def _t(a, grad=False):
    return torch.tensor(a, dtype=torch.float64, requires_grad=grad)


def _r(seed, *s):
    return np.random.default_rng(seed).standard_normal(s)


@pytest.mark.parametrize("unit", [False, True])
def test_layer_norm_and_gradients(unit):
    g, rows, D = 3, 4, 11
    x, w, b, dy, dres = _r(1, g * rows, D) * 3 + 1, _r(2, g, D), _r(3, g, D), _r(4, g * rows, D), _r(5, g * rows, D)
    y, stats = ob.layer_norm(x, w, b, rows, unit, 1e-6)
    tx, tw, tb = _t(x, True), _t(w, True), _t(b, True)
    ty = torch.cat([F.layer_norm(tx[i * rows:(i + 1) * rows], (D,), tw[i] + (1 if unit else 0), tb[i], 1e-6) for i in range(g)])
    assert np.allclose(y, ty.detach().numpy(), rtol=1e-12, atol=1e-12)
    ty.backward(_t(dy))
    dx, dw, db = ob.layer_norm_bwd(x, dy, stats, w, rows, unit, dres)
    assert np.allclose(dx - dres, tx.grad.numpy(), atol=1e-12)
    assert np.allclose(dw, tw.grad.numpy(), atol=1e-12) and np.allclose(db, tb.grad.numpy(), atol=1e-12)
    e = 1e-6                                                       # and against differences
    for i, j in ((0, 0), (5, 7), (11, 10)):
        xp, xm = x.copy(), x.copy()
        xp[i, j] += e; xm[i, j] -= e
        num = ((ob.layer_norm(xp, w, b, rows, unit)[0] - ob.layer_norm(xm, w, b, rows, unit)[0]) * dy).sum() / (2 * e)
        assert abs(num - (dx - dres)[i, j]) < 1e-7


@pytest.mark.parametrize("pairing", ["interleaved", "halves"])
@pytest.mark.parametrize("joint", [False, True])
def test_rope_axes(pairing, joint):
    x, axes = _r(1, 2, 6, 3, 14), (4, 6, 2)
    pos = np.stack([np.arange(6), 10.0 - np.arange(6), np.arange(6) * 0.5], 1)
    y = ob.rope_axes(x, pos, axes, 100.0, pairing, joint)
    assert np.array_equal(y[..., 12:], x[..., 12:])                # behind the rotated elements
    assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))         # a rotation
    assert np.allclose(ob.rope_axes(y, pos, axes, 100.0, pairing, joint, inverse=True), x)
    # products of two rotated heads depend on the difference of the positions alone
    q, k = _r(2, 1, 6, 1, 12), _r(3, 1, 6, 1, 12)
    q[:] = q[:, :1]; k[:] = k[:, :1]
    rq, rk = ob.rope_axes(q, pos, axes, 100.0, pairing, joint), ob.rope_axes(k, pos + 3.0, axes, 100.0, pairing, joint)
    d = (rq * rk).sum(-1).ravel()
    assert np.allclose(d, d[0])
    # one axis, interleaved: multiplication by exp(i t) of the pairs read as complex numbers
    one = ob.rope_axes(x[..., :4], pos[:, :1], (4,), 10000.0)
    z = x[..., 0:4:2] + 1j * x[..., 1:4:2]
    zt = z * np.exp(1j * pos[None, :, None, :1] * np.array([1.0, 0.01]))
    assert np.allclose(one[..., 0::2], zt.real) and np.allclose(one[..., 1::2], zt.imag)
    # the inverse is the gradient: <dy, J dx> = <J^T dy, dx> for a linear map
    dy = _r(4, *x.shape)
    back = ob.rope_axes(dy, pos, axes, 100.0, pairing, joint, inverse=True)
    assert np.isclose((dy * y).sum(), (back * x).sum())


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gated_linear_and_gradients(act):
    M, Fd, K = 5, 6, 4
    x, w, b, dh = _r(1, M, K), _r(2, 2 * Fd, K), _r(3, 2 * Fd), _r(4, M, Fd)
    h, z = ob.gated_linear(x, w, b, act)
    tx, tw, tb = _t(x, True), _t(w, True), _t(b, True)
    tz = F.linear(tx, tw, tb)
    th = (F.silu(tz[:, :Fd]) if act == "silu" else F.gelu(tz[:, :Fd], approximate="tanh")) * tz[:, Fd:]
    assert np.allclose(h, th.detach().numpy()) and np.allclose(z, tz.detach().numpy())
    th.backward(_t(dh))
    dx, dw, db = ob.gated_linear_bwd(x, w, z, dh, act)
    assert np.allclose(dx, tx.grad.numpy()) and np.allclose(dw, tw.grad.numpy()) and np.allclose(db, tb.grad.numpy())
    e = 1e-6
    for i, j in ((0, 0), (3, 2), (11, 1)):
        wp, wm = w.copy(), w.copy()
        wp[i, j] += e; wm[i, j] -= e
        num = ((ob.gated_linear(x, wp, b, act)[0] - ob.gated_linear(x, wm, b, act)[0]) * dh).sum() / (2 * e)
        assert abs(num - dw[i, j]) < 1e-6 * max(1, abs(num))
