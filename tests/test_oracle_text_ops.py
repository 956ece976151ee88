"""The fp64 definitions of the root-mean-square norm and of the attention to an encoder's states, pinned against torch functions,
automatic differentiation and differences."""
import numpy as np
import pytest
import torch

import synth
from oracle import block_ops as ob


def _t(a):
    return torch.from_numpy(np.asarray(a, np.float64)).requires_grad_(True)


def test_e4m3_is_torchs():
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    fine = np.sort(every[np.isfinite(every)])
    assert np.array_equal(ob.round_e4m3(fine), fine) and fine[-1] == 448.0
    v = np.concatenate([synth.normal(1, 1, (4000,)) * s for s in (1e-3, 1e-2, 1.0, 100.0)] + [(fine[1:] + fine[:-1]) / 2, [0.0, 1000.0, -1e9]])
    v = v.astype(np.float32)
    torch8 = torch.from_numpy(np.clip(v, -448, 448)).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ob.round_e4m3(v), torch8)
    assert np.isnan(ob.round_e4m3([np.nan])).all()


@pytest.mark.parametrize("unit", [False, True])
def test_rms_norm(unit):
    M, D, rows = 12, 37, 4
    x, res, w = synth.normal(2, 1, (M, D)), synth.normal(2, 2, (M, D)), synth.normal(2, 3, (3, D))
    xt, rt, wt = _t(x), _t(res), _t(w)
    gain = wt.repeat_interleave(rows, 0) + (1.0 if unit else 0.0)
    ht = xt + rt
    y = torch.nn.functional.rms_norm(ht, (D,), eps=1e-5) * gain
    yo, h, r = ob.rms_norm(x, w, res, rows, unit, 1e-5)
    assert np.allclose(y.detach().numpy(), yo, rtol=1e-12, atol=1e-13)
    dy, dres = synth.normal(2, 4, (M, D)).astype(np.float64), synth.normal(2, 5, (M, D)).astype(np.float64)
    gx, gr, gw = torch.autograd.grad((y * torch.from_numpy(dy)).sum() + (ht * torch.from_numpy(dres)).sum(), (xt, rt, wt))
    dx, dw = ob.rms_norm_bwd(h, dy, r, w, rows, unit, dres)
    assert np.allclose(gx, dx, rtol=1e-11, atol=1e-12) and np.allclose(gr, dx, rtol=1e-11, atol=1e-12) and np.allclose(gw, dw, rtol=1e-11, atol=1e-12)
    # and differences along one direction
    t = 1e-6
    u = synth.normal(2, 6, (M, D)).astype(np.float64)
    f = lambda z: (ob.rms_norm(z, w, res, rows, unit, 1e-5)[0] * dy).sum() + ((z + res) * dres).sum()
    assert np.isclose((f(x + t * u) - f(x - t * u)) / (2 * t), (dx * u).sum(), rtol=1e-6)


def test_quantise():
    y = synth.normal(3, 1, (5, 300)).astype(np.float64)
    y[2] = 0.0
    for block in (None, 128):
        q, s = ob.quantise(y, block)
        n = 300 if block is None else block
        assert s.shape == (5, -(-300 // n)) and (s[2] == 1.0).all()
        back = q * np.repeat(s, n, 1)[:, :300]
        assert (np.abs(back - y) <= np.maximum(2.0 ** -4 * np.abs(y), np.repeat(s, n, 1)[:, :300] * 2.0 ** -10) * (1 + 1e-12)).all()
        assert np.abs(q).max() == 448.0


def test_cross_attention():
    n_seq, n_q, heads, kvh, d = 4, 5, 4, 2, 6
    lens = [7, 0, 3]
    ks = [synth.normal(4, 10 + e, (n, kvh, d)).astype(np.float64) for e, n in enumerate(lens)]
    vs = [synth.normal(4, 20 + e, (n, kvh, d)).astype(np.float64) for e, n in enumerate(lens)]
    counts = [np.array([1, 1, 0, 1, 1, 0, 1], bool), np.zeros(0, bool), np.ones(3, bool)]
    enc_of = [0, 2, 0, 1]
    q, g = synth.normal(4, 1, (n_seq, n_q, heads, d)).astype(np.float64), synth.normal(4, 2, (n_seq, n_q, heads, d)).astype(np.float64)
    out, lse = ob.cross_attention(q, ks, vs, counts, enc_of, 0.3)
    assert (out[3] == 0).all() and np.isneginf(lse[3]).all()
    qt, kt, vt = _t(q), [_t(k) for k in ks], [_t(v) for v in vs]
    total = 0.0
    for s, e in enumerate(enc_of[:3]):
        kk, vv = (x[e][torch.from_numpy(counts[e])].repeat_interleave(heads // kvh, 1).transpose(0, 1) for x in (kt, vt))
        o = torch.nn.functional.scaled_dot_product_attention(qt[s].transpose(0, 1), kk, vv, scale=0.3)
        assert np.allclose(o.detach().transpose(0, 1).numpy(), out[s], rtol=1e-12, atol=1e-13)
        S = 0.3 * qt[s].transpose(0, 1) @ kk.transpose(1, 2)
        assert np.allclose(torch.logsumexp(S, 2).detach().numpy(), lse[s], rtol=1e-12)
        total = total + (o.transpose(0, 1) * torch.from_numpy(g[s])).sum()
    grads = torch.autograd.grad(total, [qt, kt[0], kt[2], vt[0], vt[2]])
    dq, dk, dv, mq, mk, mv = ob.cross_attention_bwd(q, ks, vs, counts, enc_of, 0.3, out, lse, g)
    for got, want in zip((dq, dk[0], dk[2], dv[0], dv[2]), grads):
        assert np.allclose(got, want.numpy(), rtol=1e-11, atol=1e-12)
    assert (dq[3] == 0).all() and (dk[0][2] == 0).all() and (dv[0][5] == 0).all()
    assert (mq >= np.abs(dq) - 1e-12).all() and all((a >= np.abs(b) - 1e-12).all() for a, b in zip(mk + mv, dk + dv))
    # differences along one direction of everything
    t, seed = 1e-6, 30
    uq = synth.normal(4, seed, q.shape).astype(np.float64)
    uk = [synth.normal(4, seed + 1 + e, k.shape).astype(np.float64) for e, k in enumerate(ks)]
    f = lambda z: (ob.cross_attention(q + z * uq, [k + z * u for k, u in zip(ks, uk)], [v - z * u for v, u in zip(vs, uk)], counts, enc_of, 0.3)[0] * g).sum()
    want = (dq * uq).sum() + sum((a * u).sum() - (b * u).sum() for a, b, u in zip(dk, dv, uk))
    assert np.isclose((f(t) - f(-t)) / (2 * t), want, rtol=1e-6)
