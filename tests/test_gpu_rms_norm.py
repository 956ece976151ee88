"""op_rms_norm and its backward pass against the fp64 definitions.

Tolerances (u = 2^-24).  A fp32 sum over a row adds at most 64 terms one behind the other (16 per lane, 5 exchanges, 16 warps), all of
them positive: r is off by 34 u (half the sum's relative error, and 1 / sqrt's two units).  A rounded result is off by half a step of
its type, eps / 2.  Column sums are off by (rows + 24) u of the sum of magnitudes whatever their order.
8-bit results: a scale is off by (36 + 4) u; q s is off by half a step of what it stands for, 2^-4 of the value or (below the smallest
normal number) 2^-10 of the scale, plus those 40 u."""
import numpy as np
import pytest
import torch

import synth
from oracle import block_ops as ob

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _half(dt):
    return torch.finfo(DT[dt]).eps / 2


def _mat(seed, role, shape, dt, scale=1.0, pad=0):
    """A tensor on the GPU inside rows of D + pad elements (NaN between them), and its values in fp64."""
    a = (synth.normal(seed, role, shape) * np.float32(scale)).astype(np.float32)
    full = torch.full((*shape[:-1], shape[-1] + pad), float("nan"), dtype=DT[dt], device="cuda")
    full[..., :shape[-1]] = torch.from_numpy(a).to(DT[dt])
    t = full[..., :shape[-1]]
    return t, t.double().cpu().numpy()


def _near(t, want, tol):
    return (np.abs(t.double().cpu().numpy().reshape(want.shape) - want) <= tol + 1e-37).all()


SHAPES = [  # groups, rows per group, D, extra elements between rows
    (1, 1, 1, 0), (1, 5, 2, 0), (1, 9, 8, 0), (3, 7, 40, 8), (2, 130, 256, 0), (4, 33, 384, 0), (1, 17, 511, 3), (1, 40, 512, 0), (1, 19, 513, 0),
    (3, 5, 520, 0), (2, 50, 1001, 0), (6, 41, 1152, 0), (1, 600, 1152, 40), (300, 1, 1152, 0), (700, 1, 72, 0), (1, 6, 2048, 0), (1, 7, 2056, 0),
    (2, 50, 870, 0), (1, 33, 1154, 2), (2, 20, 384, 2), (1, 20, 384, 1), (2, 3, 4608, 0), (1, 3, 8191, 0), (1, 2, 8192, 0), (1, 3000, 24, 0), (1, 3, 4096, 0),
    (1, 9, 768, 0), (2, 9, 1024, 0), (1, 5, 129, 0), (1, 20, 130, 0), (1, 3, 1028, 0),
]


@pytest.mark.parametrize("xd,rd,yd", [("fp32", None, "fp32"), ("bf16", None, "bf16"), ("bf16", "fp32", "bf16"), ("bf16", "bf16", "fp32"), ("fp32", "fp32", "bf16"),
                                      ("fp32", "bf16", "fp32")])
@pytest.mark.parametrize("g,rows,D,pad", SHAPES)
def test_forward_and_backward(g, rows, D, pad, xd, rd, yd):
    import paper_2511_20390_b200 as free
    M, seed, unit = g * rows, g + 10 * rows + D, g > 1
    x, xf = _mat(seed, 1, (M, D), xd, 1.5, pad)
    res, rf = (None, None) if rd is None else _mat(seed, 2, (M, D), rd, 2.0, pad)
    w = 0.3 * synth.normal(seed, 3, (g, D))
    wt = torch.from_numpy(w).cuda()
    got = free.op_rms_norm(x, wt, residual=res, rows_per_group=rows, unit_offset=unit, out_dtype=DT[yd], want_rstd=True)
    yo, ho, ro = ob.rms_norm(xf, w, rf, rows, unit)
    assert _near(got.rstd, ro, 36 * U * ro) and got.scales is None
    hmag = np.abs(xf) + (0 if rf is None else np.abs(rf))          # the sum is rounded once, half a unit of itself
    wr = np.abs(np.repeat(w.astype(np.float64), rows, 0) + (1.0 if unit else 0.0))
    assert _near(got.y, yo, U * (40 * np.abs(yo) + 2 * ro[:, None] * wr * hmag) + _half(yd) * np.abs(yo) * (1 + 1e-3))
    if rd is None:
        assert got.residual is None
        h, hf = x, xf
    else:
        h, hf = got.residual, got.residual.double().cpu().numpy()
        assert h.dtype == DT[rd] and _near(h, ho, U * np.abs(ho) + _half(rd) * np.abs(ho) * (1 + 1e-3))
    # backward, from the h and r that the call returned
    hd = {torch.float32: "fp32", torch.bfloat16: "bf16"}[h.dtype]
    dy, dyf = _mat(seed, 4, (M, D), yd, 0.2, pad)
    dres, dresf = (None, None) if rd is None else _mat(seed, 5, (M, D), hd, 0.2)
    rg = got.rstd.double().cpu().numpy()
    dx, dw = free.op_rms_norm_bwd(h, dy, got.rstd, wt, rows_per_group=rows, unit_offset=unit, dres=dres)
    dxo, dwo = ob.rms_norm_bwd(hf, dyf, rg, w, rows, unit, dresf)
    xh, v = np.abs(hf) * rg[:, None], np.abs(dyf) * wr
    mean = (v * xh).mean(1, keepdims=True)
    tol = rg[:, None] * U * (8 * v + 76 * xh * mean) + 3 * U * ((0 if dresf is None else np.abs(dresf)) + np.abs(dxo))
    assert dx.dtype == h.dtype and _near(dx, dxo, tol + _half(hd) * np.abs(dxo) * (1 + 1e-3))
    assert _near(dw, dwo, (rows + 24) * U * (np.abs(dyf) * xh).reshape(g, rows, D).sum(1))
    again = free.op_rms_norm_bwd(h, dy, got.rstd, wt, rows_per_group=rows, unit_offset=unit, dres=dres)
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])


@pytest.mark.parametrize("xd,rd", [("bf16", "bf16"), ("bf16", "fp32"), ("fp32", None), ("bf16", None)])
@pytest.mark.parametrize("block", [None, 128])
@pytest.mark.parametrize("M,D,pad", [(1, 1, 0), (5, 72, 0), (3, 127, 0), (40, 128, 0), (33, 384, 0), (7, 511, 0), (2, 700, 4), (600, 1152, 0), (3, 1001, 0), (9, 4096, 0),
                                     (4, 5000, 0), (2, 8191, 0), (2, 8192, 0), (20, 1100, 0)])
def test_8_bit_results(M, D, pad, block, xd, rd):
    import paper_2511_20390_b200 as free
    x, xf = _mat(M + D, 1, (M, D), xd, 1.5, pad)
    res, rf = (None, None) if rd is None else _mat(M + D, 2, (M, D), rd, 2.0)
    w = 1 + 0.3 * synth.normal(M + D, 3, (1, D))
    got = free.op_rms_norm(x, torch.from_numpy(w).cuda()[0], residual=res, out_dtype=torch.float8_e4m3fn, scale_block=block)
    yo, ho, ro = ob.rms_norm(xf, w, rf)
    n = D if block is None else block
    _, so = ob.quantise(yo, block)
    assert got.y.dtype == torch.float8_e4m3fn and got.scales.shape == so.shape and got.rstd is None
    # where the sum cancels, its own half unit is what the largest value is off by
    hm = ro[:, None] * np.abs(w) * (np.abs(xf) + (0 if rf is None else np.abs(rf))) * 2 * U
    slack = np.stack([hm[:, i * n:(i + 1) * n].max(1) for i in range(so.shape[1])], 1) / 448
    assert _near(got.scales, so, 42 * U * so + slack)
    S = np.repeat(so, n, 1)[:, :D]
    back = got.y.double().cpu().numpy() * np.repeat(got.scales.double().cpu().numpy(), n, 1)[:, :D]
    assert (np.abs(back - yo) <= np.maximum(2.0 ** -4 * np.abs(yo), S * 2.0 ** -10) + 100 * U * np.abs(yo) + hm + 448 * 42 * U * S * 2.0 ** -4).all()
    if rd is not None:
        assert _near(got.residual, ho, U * np.abs(ho) + _half(rd) * np.abs(ho) * (1 + 1e-3))


@pytest.mark.parametrize("xd,yd", [("fp32", "bf16"), ("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp32")])
@pytest.mark.parametrize("tokens,H,D", [(1, 1, 8), (3, 6, 64), (50, 16, 72), (7, 3, 33), (200, 12, 128), (5, 2, 127), (33, 5, 96), (9, 1, 40), (700, 40, 20), (17, 7, 80), (5, 3, 200)])
def test_heads_inside_a_packed_projection(tokens, H, D, xd, yd):
    import paper_2511_20390_b200 as free
    seed = tokens + H + D
    full, _ = _mat(seed, 1, (tokens, 3, H, D), xd, 1.5)
    x = full[:, 1]
    xf = x.double().cpu().numpy().reshape(-1, D)
    w = 0.3 * synth.normal(seed, 2, (1, D))
    wt = torch.from_numpy(w).cuda()
    before = full.clone()
    got = free.op_rms_norm(x, wt[0], unit_offset=True, out_dtype=DT[yd], want_rstd=True)
    yo, _, ro = ob.rms_norm(xf, w, None, None, True)
    assert got.y.shape == x.shape and _near(got.y, yo, 40 * U * np.abs(yo) + _half(yd) * np.abs(yo) * (1 + 1e-3)) and _near(got.rstd, ro, 36 * U * ro)
    if xd == yd:                                                   # in place: the heads beside them stay as they are
        free.op_rms_norm(x, wt[0], unit_offset=True, out=x)
        assert torch.equal(x, got.y) and torch.equal(full[:, 0], before[:, 0]) and torch.equal(full[:, 2], before[:, 2])
        x.copy_(before[:, 1])
    if D > 128 and (D % 2 or D > 256):
        return
    dy, dyf = _mat(seed, 3, (tokens, 2, H, D), yd, 0.2)
    dy, dyf = dy[:, 0], dyf[:, 0].reshape(-1, D)
    dx, dw = free.op_rms_norm_bwd(x, dy, got.rstd, wt[0], unit_offset=True)
    rg = got.rstd.double().cpu().numpy()
    dxo, dwo = ob.rms_norm_bwd(xf, dyf, rg, w, None, True)
    xh, v = np.abs(xf) * rg[:, None], np.abs(dyf) * np.abs(w + 1)
    assert _near(dx, dxo, rg[:, None] * U * (8 * v + 76 * xh * (v * xh).mean(1, keepdims=True)) + 3 * U * np.abs(dxo) + _half(xd) * np.abs(dxo) * (1 + 1e-3))
    assert _near(dw, dwo, (len(xf) + 24) * U * (np.abs(dyf) * xh).sum(0, keepdims=True))


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float8_e4m3fn])
def test_zeros_infinities_and_nan(out):
    import paper_2511_20390_b200 as free
    x = torch.ones(5, 300, device="cuda")
    x[1] = 0
    x[2, 7] = float("nan")
    x[3, 299] = float("inf")
    x[4] = 1e-30
    r = free.op_rms_norm(x, out_dtype=out, want_rstd=True)
    y = r.y.float()
    assert torch.isfinite(y[0]).all() and (y[1] == 0).all() and torch.isnan(y[2]).all()
    assert torch.isnan(y[3, 299]) and torch.isnan(r.rstd[2]) and r.rstd[3] == 0
    if out == torch.float8_e4m3fn:
        assert r.scales[1] == 1 and torch.isnan(r.scales[2]).all()
        s = free.op_rms_norm(x, out_dtype=out, scale_block=128).scales
        assert torch.isnan(s[2, :]).all() and torch.isfinite(s[0]).all()


def test_in_place_and_missing_parts():
    import paper_2511_20390_b200 as free
    for D in (72, 1152, 1001, 4096):
        x, _ = _mat(5, 1, (37, D), "bf16")
        res, _ = _mat(5, 2, (37, D), "bf16")
        a = free.op_rms_norm(x, residual=res)
        x2, r2 = x.clone(), res.clone()
        b = free.op_rms_norm(x2, residual=r2, out=x2, residual_out=r2)
        assert b.y is x2 and b.residual is r2 and torch.equal(a.y, x2) and torch.equal(a.residual, r2)
        w = torch.ones(D, device="cuda")
        assert torch.equal(free.op_rms_norm(x).y, free.op_rms_norm(x, w).y) and torch.equal(free.op_rms_norm(x, w - 1, unit_offset=True).y, free.op_rms_norm(x).y)
        one = free.op_rms_norm(x, want_rstd=True)
        dx, dw = free.op_rms_norm_bwd(x, res, one.rstd, want_dweight=False)
        assert dw is None
        got = free.op_rms_norm_bwd(x, res, one.rstd, dx=x)[0]
        assert got is x and torch.equal(dx, x)
    e = torch.empty(0, 64, device="cuda")
    r = free.op_rms_norm(e, residual=e.clone(), want_rstd=True)
    assert r.y.shape == (0, 64) and r.rstd.shape == (0,)
    dx, dw = free.op_rms_norm_bwd(e, e.clone(), r.rstd)
    assert (dw == 0).all()
