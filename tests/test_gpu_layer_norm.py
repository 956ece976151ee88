"""free_op_layer_norm and its backward pass against the fp64 definitions.

Tolerances (u = 2^-24): a fp32 sum over a row adds at most 64 terms one behind the other (8 or 16 per lane, 5 exchanges, 32
warps), so it is off by at most 64 u sum|.|; 1 / sqrt is good to 2 units; a rounded output is off by at most half a step of its
type, eps / 2 relative to the value.  Column sums are off by at most (rows + 20) u sum|.| whatever their order."""
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


def _mat(seed, role, M, D, dt, scale=1.0, shift=0.0, pad=0):
    """[M, D] on the GPU inside rows of D + pad elements (NaN between them), and its values in fp64."""
    a = (synth.normal(seed, role, (M, D)) * np.float32(scale) + np.float32(shift)).astype(np.float32)
    full = torch.full((M, D + pad), float("nan"), dtype=DT[dt], device="cuda")
    full[:, :D] = torch.from_numpy(a).to(DT[dt])
    t = full[:, :D]
    return t, t.double().cpu().numpy()


def _tab(seed, role, g, D):
    a = 0.3 * synth.normal(seed, role, (g, D))
    return torch.from_numpy(a).cuda(), a.astype(np.float64)


def _per_row(v, rows):
    return np.repeat(v, rows, 0)


def _fwd_tol(x, stats, w_rows, b_rows, y, out):
    mu, r = stats[:, :1], stats[:, 1:]
    xh = np.abs(x - mu) * r
    d_xh = U * (64 * r * np.abs(x).mean(1, keepdims=True) + 72 * xh)
    return d_xh * np.abs(w_rows) + 4 * U * (xh * np.abs(w_rows) + np.abs(b_rows)) + _half(out) * np.abs(y) * (1 + 1e-3) + 1e-37


SHAPES = [  # groups, rows per group, D, extra elements between rows of x
    (1, 1, 1, 0), (1, 5, 2, 0), (1, 9, 8, 0), (3, 7, 40, 8), (2, 130, 256, 0), (4, 33, 384, 0), (1, 17, 511, 3), (1, 40, 512, 0),
    (1, 19, 513, 0), (3, 5, 520, 0), (2, 50, 1001, 0), (6, 41, 1152, 0), (1, 600, 1152, 40), (300, 1, 1152, 0), (700, 1, 72, 0),
    (1, 6, 2048, 0), (1, 7, 2056, 0), (2, 50, 870, 0), (1, 33, 1154, 2), (1, 9, 4602, 0), (2, 20, 384, 2), (1, 20, 384, 1), (1, 10, 2304, 2), (1, 300, 6, 0), (2, 3, 4608, 0), (1, 3, 8191, 0), (1, 2, 8192, 0), (1, 3000, 24, 0),
]


@pytest.mark.parametrize("xd,yd", [("fp32", "bf16"), ("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp32")])
@pytest.mark.parametrize("g,rows,D,pad", SHAPES)
def test_forward_and_backward(g, rows, D, pad, xd, yd):
    import paper_2511_20390_b200 as free
    M, seed = g * rows, g + 10 * rows + D
    x, xf = _mat(seed, 1, M, D, xd, 1.5, 0.7, pad)
    unit = g > 1
    w, wf = _tab(seed, 2, g, D)
    b, bf = _tab(seed, 3, g, D)
    y, stats = free.op_layer_norm(x, w, b, rows_per_group=rows, unit_offset=unit, out_dtype=DT[yd], want_stats=True)
    yo, so = ob.layer_norm(xf, wf, bf, rows, unit)
    wr, br = _per_row(wf, rows) + (1.0 if unit else 0.0), _per_row(bf, rows)
    sg = stats.double().cpu().numpy()
    assert (np.abs(sg[:, 0] - so[:, 0]) <= 66 * U * np.abs(xf).mean(1) + 1e-37).all()
    # r: half the variance's relative error (squared deviations, and the mean's own error, of second order) and 1 / sqrt's
    assert (np.abs(sg[:, 1] - so[:, 1]) <= so[:, 1] * (72 * U + (66 * U * np.abs(xf).mean(1) * so[:, 1]) ** 2)).all()
    assert (np.abs(y.double().cpu().numpy() - yo) <= _fwd_tol(xf, so, wr, br, yo, yd)).all()

    # backward, from the statistics that the call returned
    dy, dyf = _mat(seed, 4, M, D, yd, 0.2, 0.01, pad)
    res, resf = _mat(seed, 5, M, D, xd, 0.2)
    dx, dw, db = free.op_layer_norm_bwd(x, dy, stats, w, rows_per_group=rows, unit_offset=unit, dres=res)
    dxo, dwo, dbo = ob.layer_norm_bwd(xf, dyf, sg, wf, rows, unit, resf)
    mu, r = sg[:, :1], sg[:, 1:]
    xh, v = np.abs(xf - mu) * r, np.abs(dyf * wr)
    mean = lambda a: a.mean(1, keepdims=True)
    tol = r * U * (8 * (v + mean(v) + xh * mean(v * xh)) + 64 * mean(v) + 70 * xh * mean(v * xh)) + 3 * U * (np.abs(resf) + np.abs(dxo))
    assert (np.abs(dx.double().cpu().numpy() - dxo) <= tol + _half(xd) * np.abs(dxo) * (1 + 1e-3) + 1e-37).all()
    cols = lambda a: a.reshape(g, rows, D).sum(1)
    assert (np.abs(dw.double().cpu().numpy() - dwo) <= (rows + 24) * U * cols(np.abs(dyf) * xh) + 1e-37).all()
    assert (np.abs(db.double().cpu().numpy() - dbo) <= (rows + 20) * U * cols(np.abs(dyf)) + 1e-37).all()
    # the same bits again
    again = free.op_layer_norm_bwd(x, dy, stats, w, rows_per_group=rows, unit_offset=unit, dres=res)
    assert all(torch.equal(p, q) for p, q in zip((dx, dw, db), again))


def test_a_large_mean_cancels_nothing():
    import paper_2511_20390_b200 as free
    for D in (96, 1152, 1001):
        x, xf = _mat(3, 1, 64, D, "fp32", 1.0, 3.0e3)
        y = free.op_layer_norm(x)
        yo, so = ob.layer_norm(xf)
        assert (np.abs(y.double().cpu().numpy() - yo) <= _fwd_tol(xf, so, 1.0, 0.0, yo, "fp32")).all()


@pytest.mark.parametrize("xd,yd", [("fp32", "bf16"), ("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp32")])
@pytest.mark.parametrize("g,rows,D,pad", [
    (1, 1, 1, 0), (3, 1, 2, 0), (5, 2, 3, 1), (2, 37, 8, 0), (1, 130, 30, 2), (9, 7, 32, 0), (1, 517, 33, 0), (4, 129, 40, 8),
    (1, 1000, 62, 0), (70, 3, 64, 0), (2, 700, 64, 4), (1, 640, 65, 1), (3, 200, 100, 0), (1, 20011, 64, 0), (300, 65, 96, 0),
    (1, 2500, 110, 0), (2, 300, 126, 2), (1, 333, 127, 0), (3, 257, 128, 0), (1, 150, 129, 0), (2, 90, 200, 0), (1, 77, 255, 0),
])
def test_narrow_rows(g, rows, D, pad, xd, yd):
    """Up to 128 columns several rows share a warp: groups that begin and end inside one, runs that end inside one."""
    test_forward_and_backward(g, rows, D, pad, xd, yd)


@pytest.mark.parametrize("D", [8, 33, 512, 1152])
def test_defaults_shared_tables_and_missing_parts(D):
    import paper_2511_20390_b200 as free
    x, xf = _mat(5, 1, 12, D, "fp32", 1.0)
    dy, dyf = _mat(5, 2, 12, D, "fp32", 1.0)
    w, wf = _tab(5, 3, 1, D)
    assert torch.equal(free.op_layer_norm(x, w[0]), free.op_layer_norm(x, w, rows_per_group=4))     # one row for all groups
    assert torch.equal(free.op_layer_norm(x, w * 0 + 1, w * 0), free.op_layer_norm(x))
    y, stats = free.op_layer_norm(x, want_stats=True)
    dx, dw, db = free.op_layer_norm_bwd(x, dy, stats, rows_per_group=4)
    assert dw.shape == (3, D) and db.shape == (3, D)
    dxo, dwo, dbo = ob.layer_norm_bwd(xf, dyf, stats.double().cpu().numpy(), None, 4)
    assert np.abs(dw.double().cpu().numpy() - dwo).max() < 1e-5 and np.abs(db.double().cpu().numpy() - dbo).max() < 1e-5
    only, no_w, no_b = free.op_layer_norm_bwd(x, dy, stats, rows_per_group=4, want_dweight=False, want_dbias=False)
    assert no_w is None and no_b is None and torch.equal(only, dx)
    one = free.op_layer_norm_bwd(x, dy, stats, rows_per_group=4, want_dweight=False)
    assert one[1] is None and torch.equal(one[2], db)
    # tables inside a wider one, as an adaLN projection leaves them
    table = torch.from_numpy(synth.normal(5, 6, (3, 6 * D))).cuda()
    shift, scale = table[:, :D], table[:, D:2 * D]
    ref = free.op_layer_norm(x, scale.contiguous(), shift.contiguous(), rows_per_group=4, unit_offset=True)
    assert torch.equal(free.op_layer_norm(x, scale, shift, rows_per_group=4, unit_offset=True), ref)
    # the same formula as the modulated norm that the passes use
    mod = free.op_ln_modulate(x, shift, scale, 4)
    assert (mod - ref).abs().max().item() <= 64 * U * 4 * ref.abs().max().item()


def test_empty_batches():
    import paper_2511_20390_b200 as free
    x = torch.empty(0, 1152, device="cuda")
    y, stats = free.op_layer_norm(x, want_stats=True)
    assert y.shape == (0, 1152) and stats.shape == (0, 2)
    dx, dw, db = free.op_layer_norm_bwd(x, x, stats)
    assert dx.shape == (0, 1152) and not dw.any() and not db.any() and dw.shape == (1, 1152)


def test_in_place_rows_between_and_bad_values():
    import paper_2511_20390_b200 as free
    for D, pad in ((1152, 8), (384, 16), (77, 3)):
        x, xf = _mat(7, 1, 20, D, "fp32", 1.0, 0.0, pad)
        ref, stats = free.op_layer_norm(x, want_stats=True)
        dy, _ = _mat(7, 2, 20, D, "fp32")
        dref = free.op_layer_norm_bwd(x, dy, stats, dres=dy)
        # gradient written over the residual path's gradient
        buf = dy.clone()
        got = free.op_layer_norm_bwd(x, dy, stats, dres=buf, dx=buf)
        assert got[0] is buf and torch.equal(buf, dref[0]) and torch.equal(got[1], dref[1])
        # a row with an infinity and one with a NaN: those rows alone
        xb = x.clone()
        xb[3, D // 2] = float("inf"); xb[11, 0] = float("nan")
        yb = free.op_layer_norm(xb)
        keep = [i for i in range(20) if i not in (3, 11)]
        assert torch.equal(yb[keep], ref[keep]) and torch.isnan(yb[[3, 11]]).all()
        # in place; what lies between the rows stays
        base = x.as_strided((20, D + pad), (D + pad, 1))
        free.op_layer_norm(x, out=x)
        assert torch.equal(x, ref) and torch.isnan(base[:, D:]).all()


@pytest.mark.parametrize("D,pad", [(6, 2), (32, 0), (64, 8), (96, 3), (127, 0), (200, 4), (255, 1)])
def test_narrow_rows_in_place_missing_parts_and_bad_values(D, pad):
    import paper_2511_20390_b200 as free
    M, T = 203, 29
    x, _ = _mat(17, 1, M, D, "bf16", 1.0, 0.2, pad)
    dy, _ = _mat(17, 2, M, D, "bf16", 1.0, 0.0, pad)
    w, _ = _tab(17, 3, M // T, D)
    b, _ = _tab(17, 4, M // T, D)
    ref, st = free.op_layer_norm(x, w, b, rows_per_group=T, want_stats=True)
    dref = free.op_layer_norm_bwd(x, dy, st, w, rows_per_group=T)
    # either gradient of the tables alone, or none
    for ww, wb in ((True, False), (False, True), (False, False)):
        got = free.op_layer_norm_bwd(x, dy, st, w, rows_per_group=T, want_dweight=ww, want_dbias=wb)
        assert torch.equal(got[0], dref[0]) and (got[1] is None) != ww and (got[2] is None) != wb
        assert (not ww or torch.equal(got[1], dref[1])) and (not wb or torch.equal(got[2], dref[2]))
    # either table alone
    one = torch.ones_like(w)
    assert torch.equal(free.op_layer_norm(x, None, b, rows_per_group=T), free.op_layer_norm(x, one, b, rows_per_group=T))
    assert torch.equal(free.op_layer_norm(x, w, rows_per_group=T), free.op_layer_norm(x, w, torch.zeros_like(b), rows_per_group=T))
    # a row with an infinity and one with a NaN, beside good ones in the same warp
    xb = x.clone()
    xb[3, D // 2] = float("inf"); xb[101, 0] = float("nan"); xb[M - 1, D - 1] = float("-inf")
    yb = free.op_layer_norm(xb, w, b, rows_per_group=T)
    keep = [i for i in range(M) if i not in (3, 101, M - 1)]
    assert torch.equal(yb[keep], ref[keep]) and torch.isnan(yb[[3, 101, M - 1]]).all()
    # dx over each of its inputs, then y over x; what lies between the rows stays
    for which in (0, 1):
        a, g = (torch.full((M, D + 4), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        a[:, :D], g[:, :D] = x, dy
        dst, beside = (a, g)[which], torch.full_like(a, 7.0)
        # (a result of the same strides: they may choose another width of access, another order of the same sums)
        want = free.op_layer_norm_bwd(a[:, :D], g[:, :D], st, w, rows_per_group=T, dx=beside[:, :D])
        got = free.op_layer_norm_bwd(a[:, :D], g[:, :D], st, w, rows_per_group=T, dx=dst[:, :D])
        assert torch.equal(dst, beside) and (dst[:, D:] == 7.0).all() and torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])
    base = x.as_strided((M, D + pad), (D + pad, 1))
    free.op_layer_norm(x, w, b, rows_per_group=T, out=x)
    assert torch.equal(x, ref) and torch.isnan(base[:, D:]).all()


def test_rows_far_apart():
    # two rows more than 2^32 bytes apart in one allocation, in and out
    import paper_2511_20390_b200 as free
    step = (1 << 31) + 64
    buf = torch.empty(step + 1152, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((2, 1152), (step, 1))
    x.copy_(_mat(13, 1, 2, 1152, "bf16")[0])
    ref, st = free.op_layer_norm(x.contiguous(), want_stats=True)
    dref = free.op_layer_norm_bwd(x.contiguous(), ref, st)
    assert torch.equal(free.op_layer_norm(x), ref)
    got = free.op_layer_norm_bwd(x, ref, st, dx=x)
    assert torch.equal(x, dref[0]) and torch.equal(got[1], dref[1])


def test_unaligned_tables_and_gradients_over_their_inputs():
    # tables whose rows start at any element take the scalar form: another order of the same sums
    import paper_2511_20390_b200 as free
    for D in (1152, 384, 2304, 513):
        x, xf = _mat(14, 1, 30, D, "fp32")
        dy, dyf = _mat(14, 2, 30, D, "fp32")
        table = torch.from_numpy(synth.normal(14, 3, (3, 2 * D + 3))).cuda()
        w, b = table[:, 1:D + 1], table[:, D + 2:2 * D + 2]
        y, st = free.op_layer_norm(x, w, b, rows_per_group=10, want_stats=True)
        wf, bf = w.double().cpu().numpy(), b.double().cpu().numpy()
        yo, so = ob.layer_norm(xf, wf, bf, 10)
        assert (np.abs(y.double().cpu().numpy() - yo) <= _fwd_tol(xf, so, _per_row(wf, 10), _per_row(bf, 10), yo, "fp32")).all()
        for tab in (w, w.contiguous()):
            ref = free.op_layer_norm_bwd(x, dy, st, tab, rows_per_group=10)
            dwo = ob.layer_norm_bwd(xf, dyf, st.double().cpu().numpy(), wf, 10)[1]
            xh = np.abs(xf - st[:, :1].double().cpu().numpy()) * st[:, 1:].double().cpu().numpy()
            assert (np.abs(ref[1].double().cpu().numpy() - dwo) <= 34 * U * (np.abs(dyf) * xh).reshape(3, 10, D).sum(1)).all()
            for over in (x, dy):                                   # dx written over one of its inputs: the same bits
                a, g = x.clone(), dy.clone()
                dst = a if over is x else g
                got = free.op_layer_norm_bwd(a, g, st, tab, rows_per_group=10, dx=dst)
                assert torch.equal(dst, ref[0]) and torch.equal(got[1], ref[1]) and torch.equal(got[2], ref[2])


def test_a_constant_row_and_a_tiny_variance():
    import paper_2511_20390_b200 as free
    x = torch.full((4, 1152), 2.5, device="cuda")
    y, stats = free.op_layer_norm(x, want_stats=True, eps=1e-6)
    assert not y.any() and np.allclose(stats[:, 1].cpu().numpy(), 1e3, rtol=1e-6)
    y0 = free.op_layer_norm(torch.zeros(4, 40, device="cuda"), eps=1e-12)
    assert not y0.any()


def test_streams_and_graphs():
    import paper_2511_20390_b200 as free
    x, _ = _mat(9, 1, 2000, 1152, "fp32")
    dy, _ = _mat(9, 2, 2000, 1152, "bf16")
    w, _ = _tab(9, 3, 2, 1152)
    y, st = free.op_layer_norm(x, w, w, rows_per_group=1000, out_dtype=torch.bfloat16, want_stats=True)
    ref = free.op_layer_norm_bwd(x, dy, st, w, rows_per_group=1000)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = free.op_layer_norm_bwd(x, dy, st, w, rows_per_group=1000)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, got))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y2, st2 = free.op_layer_norm(x, w, w, rows_per_group=1000, out_dtype=torch.bfloat16, want_stats=True)
        got = free.op_layer_norm_bwd(x, dy, st2, w, rows_per_group=1000)
    x.mul_(2.0); dy.neg_()
    g.replay()
    torch.cuda.synchronize()
    y3, st3 = free.op_layer_norm(x, w, w, rows_per_group=1000, out_dtype=torch.bfloat16, want_stats=True)
    ref = free.op_layer_norm_bwd(x, dy, st3, w, rows_per_group=1000)
    assert torch.equal(y2, y3) and all(torch.equal(a, b) for a, b in zip(ref, got))


def test_the_tolerance_sees_one_dropped_row():
    # a mistake planted in the definition: one row of one group left out of the sums
    xf, dyf = synth.normal(1, 1, (600, 64)).astype(np.float64), synth.normal(1, 2, (600, 64)).astype(np.float64)
    _, st = ob.layer_norm(xf)
    _, dw, _ = ob.layer_norm_bwd(xf, dyf, st)
    _, less, _ = ob.layer_norm_bwd(xf[1:], dyf[1:], st[1:])
    xh = np.abs(xf - st[:, :1]) * st[:, 1:]
    assert (np.abs(dw - less) > 624 * U * (np.abs(dyf) * xh).sum(0)).any()
