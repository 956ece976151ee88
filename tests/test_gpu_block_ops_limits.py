"""Block operators at the limits of their ranges: gates far out, more column tiles than a grid dimension holds, results given by
the caller."""
import numpy as np
import pytest
import torch

from oracle import block_ops as ob

pytestmark = pytest.mark.gpu

DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_gradients_of_gates_far_out(act, dt):
    # where the activation is g or 0 its slope is 1 or 0 exactly, up to the largest gates (the square of 2e19 is past fp32)
    import paper_2511_20390_b200 as free
    far = [120.0, 1e4, 1e10, 1.5e19, 2e19, 1e25, 1e30, 3e38]
    gates = torch.tensor([-v for v in far[::-1]] + far, device="cuda").to(DT[dt])
    M, F, K, step = 5, len(gates), 8, 2.0 ** -10
    pre = torch.cat([gates, torch.ones_like(gates)]).repeat(M, 1)
    x, w = torch.ones(M, K, dtype=DT[dt], device="cuda"), torch.zeros(2 * F, K, dtype=DT[dt], device="cuda")
    w[0] = 1.0                                                     # its slope is 0, so dx is 0
    dh = torch.full((M, F), step, dtype=DT[dt], device="cuda")
    dx, dw, db = free.op_gated_linear_bwd(x, w, pre, dh, act=act)
    slope = np.concatenate([np.zeros(F // 2), np.ones(F // 2)])
    assert not np.any(ob.gate_act(act, np.array([-700.0]))[1] > 1e-300) and ob.gate_act(act, np.array([700.0]))[1] == 1.0
    assert np.array_equal(db[:F].cpu().numpy(), M * step * slope)
    assert np.array_equal(dw[:F].double().cpu().numpy(), np.repeat((M * step * slope)[:, None], K, 1))
    # five equal terms, each rounded once, and four sums: 2^-21 of them; dw is rounded to its type besides
    a = gates.double().cpu().numpy() * slope
    assert (np.abs(db[F:].double().cpu().numpy() - M * step * a) <= 2.0 ** -21 * M * step * a).all()
    half = torch.finfo(DT[dt]).eps / 2
    assert (np.abs(dw[F:].double().cpu().numpy() - (M * step * a)[:, None]) <= (2.0 ** -21 + half) * (M * step * a)[:, None]).all()
    assert not dx.any() and not torch.isnan(dx).any()


def test_fp32_columns_past_a_grid_dimension():
    # 65536 column tiles and more; a contraction of four terms: off by at most 12 units of 2^-24 of the terms' sizes, the
    # activation by (16 + 1.2 |argument|) 2^-23 besides (the bounds of the operator's other tests)
    import paper_2511_20390_b200 as free
    U = 2.0 ** -24
    g = torch.Generator(device="cuda").manual_seed(5)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    M, F, K = 26, 64 * 65536 + 5, 4                                # forward: 64 columns of each half per tile
    x, w, b = rnd(M, K), rnd(2 * F, K), rnd(2 * F)
    h, pre = free.op_gated_linear(x, w, b, want_preact=True)
    for lo, hi in ((0, 100000), (F - 100000, F)):
        rows = torch.cat([torch.arange(lo, hi), torch.arange(F + lo, F + hi)]).cuda()
        size = x.double().abs() @ w[rows].double().abs().t() + b[rows].double().abs()
        z = x.double() @ w[rows].double().t() + b[rows].double()
        assert ((pre[:, rows].double() - z).abs() <= 12 * U * size).all()
        n = hi - lo
        zg, zu = z[:, :n], z[:, n:]
        tol = 1.2 * 12 * U * size[:, :n] * (zu.abs() + 12 * U * size[:, n:]) + zg.abs() * 12 * U * size[:, n:] + (16 + 1.2 * zg.abs()) * 2 * U * (zg * zu).abs()
        assert ((h[:, lo:hi].double() - zg * torch.sigmoid(zg) * zu).abs() <= tol + 1e-37).all()
    del w, b, h, pre
    M, F, K = 3, 2, 128 * 65536 + 77                               # backward: 128 columns per tile of dx and of dw
    x, w, pre, dh = rnd(M, K), rnd(2 * F, K), rnd(M, 2 * F), rnd(M, F)
    dx, dw, db = free.op_gated_linear_bwd(x, w, pre, dh)
    zg, zu = pre[:, :F].double(), pre[:, F:].double()
    s = torch.sigmoid(zg)
    dz = torch.cat([dh.double() * zu * (s + zg * s * (1 - s)), dh.double() * zg * s], 1)
    err = (16 + 1.2 * torch.cat([zg, zg], 1).abs()) * 2 * U * torch.cat([(dh.double() * zu).abs() * (1 + 1.2 * zg.abs()), (dh.double() * zg).abs()], 1)
    for got, a, e, m in ((dx, dz, err, w), (dw, dz.t(), err.t(), x)):
        ref, size = a @ m.double(), (a.abs() + e) @ m.double().abs()
        assert ((got.double() - ref).abs() <= e @ m.double().abs() + 12 * U * size + 1e-37).all()
    assert ((db.double() - dz.sum(0)).abs() <= (err + 12 * U * dz.abs()).sum(0)).all()


def test_out_dtype_beside_out():
    import paper_2511_20390_b200 as free
    x = torch.randn(3, 64, device="cuda")
    out = torch.empty(3, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="out_dtype"):
        free.op_layer_norm(x, out=out, out_dtype=torch.float32)
    assert free.op_layer_norm(x, out=out, out_dtype=torch.bfloat16) is out
    assert torch.equal(out, free.op_layer_norm(x, out_dtype=torch.bfloat16))


def test_results_that_overlap_an_input_are_refused():
    import paper_2511_20390_b200 as free
    buf = torch.randn(200 * 64, device="cuda")
    x, dy = buf[:100 * 64].view(100, 64), torch.randn(100, 64, device="cuda")
    want, st = free.op_layer_norm(x, want_stats=True)
    kept = buf.clone()
    for at in (64, 4, 99 * 64):                                    # rows or a few elements further on
        out = buf[at:at + 100 * 64].view(100, 64)
        with pytest.raises(ValueError, match="overlap"):
            free.op_layer_norm(x, out=out)
        with pytest.raises(ValueError, match="overlap"):
            free.op_layer_norm_bwd(x, dy, st, dx=out)
        with pytest.raises(ValueError, match="overlap"):
            free.op_layer_norm_bwd(dy, x, st, dx=out)
        with pytest.raises(ValueError, match="overlap"):
            free.op_layer_norm_bwd(dy, dy, st, dres=x, dx=out)
    with pytest.raises(ValueError, match="overlap"):               # the same place, another type
        free.op_layer_norm(x, out=buf.view(torch.bfloat16)[:100 * 64].view(100, 64))
    with pytest.raises(ValueError, match="overlap"):
        free.op_layer_norm(x, buf[:64], out=x)                     # the weight is one of the rows
    pos = torch.arange(10, dtype=torch.float32, device="cuda")[:, None]
    qkv = torch.randn(2, 10, 6, 16, device="cuda")
    for lo, hi in ((1, 5), (2, 6)):
        with pytest.raises(ValueError, match="overlap"):
            free.op_rope_axes(qkv[:, :, :4], pos, (16,), out=qkv[:, :, lo:hi])
    w, h = torch.randn(2 * 64, 64, device="cuda"), torch.empty(100, 64, device="cuda")
    for out in (x, buf[64:101 * 64].view(100, 64)):
        with pytest.raises(ValueError, match="overlap"):
            free.op_gated_linear(x, w, out=out)
    with pytest.raises(ValueError, match="overlap"):
        free.op_gated_linear(x, w, out=w[:100])
    assert torch.equal(buf, kept)
    # beside one another in one buffer, and element for element over an input
    assert torch.equal(free.op_layer_norm(x, out=buf[100 * 64:].view(100, 64)), want)
    two = torch.zeros(100, 128, device="cuda")
    two[:, :64] = x
    assert torch.equal(free.op_layer_norm(two[:, :64], out=two[:, 64:]), want) and torch.equal(two[:, :64], x)
    rot = free.op_rope_axes(qkv[:, :, :2], pos, (16,))
    assert torch.equal(free.op_rope_axes(qkv[:, :, :2], pos, (16,), out=qkv[:, :, 2:4]), rot)
    assert torch.equal(free.op_rope_axes(qkv[:, :, :2], pos, (16,), out=qkv[:, :, :2]), rot)
    assert torch.equal(free.op_gated_linear(x, w, out=h), free.op_gated_linear(x, w))
    assert torch.equal(free.op_layer_norm(x, out=x), want)
