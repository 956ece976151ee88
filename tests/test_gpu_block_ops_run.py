"""The block operators together, as a rotary, gated DiT block uses them: modulated norm, projection, rotary positions in place in
the packed projection, attention, residual, modulated norm, gated layer, projection, residual; and the backward pass of the
feed-forward half.  Against the fp64 definitions."""
import numpy as np
import pytest
import torch
import torch.nn.functional as TF

import synth
from gpu_util import rms_rel
from oracle import block_ops as ob

pytestmark = pytest.mark.gpu


def _t(seed, role, shape, dt, scale=1.0):
    return torch.from_numpy((synth.normal(seed, role, shape) * np.float32(scale)).astype(np.float32)).to(dt).cuda()


def _f(t):
    return t.double().cpu().numpy()


BF, FP = (torch.bfloat16, 2e-2), (torch.float32, 2e-5)


@pytest.mark.parametrize("n_seq,side,heads,dh,dt,tol", [(2, 16, 6, 64, *BF), (2, 16, 6, 64, *FP), (1, 32, 8, 72, *BF), (1, 16, 4, 72, *FP),
                                                        (3, 5, 2, 16, *FP)])
def test_forward_block(n_seq, side, heads, dh, dt, tol):
    # 2e-2: the framework's bound for bf16 passes; fp32: sums of at most a thousand terms, a handful of them in a row
    import paper_2511_20390_b200 as free
    from paper_2511_20390_b200 import binding
    T, D = side * side, heads * dh
    F, M = 2 * D, n_seq * T
    code = binding._code(dt)
    x = _t(1, 1, (M, D), torch.float32)
    mod = _t(1, 2, (n_seq, 6 * D), torch.float32, 0.2)
    sh1, sc1, g1, sh2, sc2, g2 = mod.split(D, dim=1)
    wqkv, wo = _t(1, 3, (3 * D, D), dt, D ** -0.5), _t(1, 4, (D, D), dt, D ** -0.5)
    w12, w3 = _t(1, 5, (2 * F, D), dt, D ** -0.5), _t(1, 6, (D, F), dt, F ** -0.5)
    pos = torch.from_numpy(np.stack(np.divmod(np.arange(T), side), 1).astype(np.float32)).cuda()
    axes = (dh // 4 * 2, dh - dh // 4 * 2)
    res = x.clone()
    y = free.op_layer_norm(res, sc1, sh1, rows_per_group=T, unit_offset=True, out_dtype=dt)
    qkv = free.op_linear(y, wqkv, out_dtype=code).view(n_seq, T, 3 * heads, dh)
    qk = qkv[:, :, :2 * heads]
    free.op_rope_axes(qk, pos, axes, out=qk)
    att = free.op_attention(qkv.view(n_seq, T, 3 * D), heads)
    free.op_linear(att.view(M, D), wo, epilogue=binding.EPI_GATE_RESIDUAL, resid=res, gate=g1, rows_per_seq=T)
    y = free.op_layer_norm(res, sc2, sh2, rows_per_group=T, unit_offset=True, out_dtype=dt)
    h = free.op_gated_linear(y, w12)
    free.op_linear(h, w3, epilogue=binding.EPI_GATE_RESIDUAL, resid=res, gate=g2, rows_per_seq=T)
    assert free.op_device_error() == 0

    rep = lambda v: np.repeat(_f(v), T, 0)
    r = _f(x)
    yo, _ = ob.layer_norm(r, _f(sc1), _f(sh1), T, True)
    q = (yo @ _f(wqkv).T).reshape(n_seq, T, 3 * heads, dh)
    q[:, :, :2 * heads] = ob.rope_axes(q[:, :, :2 * heads], _f(pos), axes)
    q = torch.from_numpy(q).view(n_seq, T, 3, heads, dh).permute(2, 0, 3, 1, 4)
    ao = TF.scaled_dot_product_attention(q[0], q[1], q[2]).permute(0, 2, 1, 3).reshape(M, D).numpy()
    r = r + rep(g1) * (ao @ _f(wo).T)
    yo, _ = ob.layer_norm(r, _f(sc2), _f(sh2), T, True)
    ho, _ = ob.gated_linear(yo, _f(w12))
    r = r + rep(g2) * (ho @ _f(w3).T)
    assert rms_rel(res - x, r - _f(x)) < tol
    assert rms_rel(h, ho) < tol


@pytest.mark.parametrize("dt,tol", [(torch.bfloat16, 2e-2), (torch.float32, 1e-5)])
def test_training_step_of_the_feed_forward_half(dt, tol):
    """x -> norm -> gated layer, with the residual path's gradient: against torch autograd in fp64."""
    import paper_2511_20390_b200 as free
    n, T, D, F = 3, 70, 128, 200
    x = _t(2, 1, (n * T, D), torch.float32)
    scale, shift = _t(2, 2, (n, D), torch.float32, 0.2), _t(2, 3, (n, D), torch.float32, 0.2)
    w, b = _t(2, 4, (2 * F, D), dt, D ** -0.5), _t(2, 5, (2 * F,), torch.float32, 0.1)
    dh, dres = _t(2, 6, (n * T, F), dt, 0.1), _t(2, 7, (n * T, D), torch.float32, 0.1)
    y, st = free.op_layer_norm(x, scale, shift, rows_per_group=T, unit_offset=True, out_dtype=dt, want_stats=True)
    h, pre = free.op_gated_linear(y, w, b, want_preact=True)
    dy, dw, db = free.op_gated_linear_bwd(y, w, pre, dh)
    dx, dscale, dshift = free.op_layer_norm_bwd(x, dy, st, scale, rows_per_group=T, unit_offset=True, dres=dres)
    assert free.op_device_error() == 0
    leaves = [t.double().cpu().requires_grad_() for t in (x, scale, shift, w, b)]
    xo, sco, sho, wo, bo = leaves
    yo = TF.layer_norm(xo, (D,), eps=1e-6) * (1 + sco.repeat_interleave(T, 0)) + sho.repeat_interleave(T, 0)
    z = TF.linear(yo, wo, bo)
    ho = TF.silu(z[:, :F]) * z[:, F:]
    ho.backward(dh.double().cpu())
    for got, ref in ((h, ho.detach()), (dx - dres, xo.grad), (dscale, sco.grad), (dshift, sho.grad), (dw, wo.grad), (db, bo.grad)):
        assert rms_rel(got, ref.numpy()) < tol


def test_rotation_and_its_gradient():
    import paper_2511_20390_b200 as free
    q = _t(3, 1, (2, 49, 3, 24), torch.float32)
    dy = _t(3, 2, (2, 49, 3, 24), torch.float32)
    pos = torch.from_numpy(np.stack(np.divmod(np.arange(49), 7), 1).astype(np.float32)).cuda()
    y = free.op_rope_axes(q, pos, (12, 12), pairing="halves")
    back = free.op_rope_axes(dy, pos, (12, 12), pairing="halves", inverse=True)
    # the rotation is linear: <dy, R q> = <R^T dy, q>
    a, b = (_f(dy) * _f(y)).sum(), (_f(back) * _f(q)).sum()
    assert abs(a - b) < 1e-4 * np.abs(_f(dy) * _f(y)).sum() ** 0.5
