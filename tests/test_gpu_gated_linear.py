"""free_op_gated_linear and its backward pass against the fp64 definitions.

Tolerances (u = 2^-24).  fp32: a sum of n products is off by at most (n + 8) u sum|.| whatever its order.  bf16 on the tensor
cores: products of bf16 values are exact in fp32; the accumulator is renewed once per 16 terms, each time off by at most four
units (2^-22) of sum|.|.  dz is rounded to bf16 once for the products of the backward pass: half a step (2^-8 of the value) of
every term.  The fast logistic function is good to 8 + 1.2 |argument| units.  Outputs are rounded once to their type.
A worst-case bound over a long sum is far above what independent roundings give, so bf16 gradients are also held to 4e-3 in
the 2-norm: dz and the output are each off by 1.7e-3 of the value (root mean square), together 2.4e-3."""
import numpy as np
import pytest
import torch

import synth
from oracle import block_ops as ob

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
TINY = 1e-37


def _g(seed, role, shape, dt, scale=1.0):
    t = torch.from_numpy((synth.normal(seed, role, shape) * np.float32(scale)).astype(np.float32)).to(DT[dt]).cuda()
    return t, t.double().cpu().numpy()


def _f64(t):
    return t.double().cpu().numpy()


def _sum_err(n, dt):
    return (n + 8) * U if dt == "fp32" else (n / 16 + 4) * 4 * U


def _half(dt):
    return torch.finfo(DT[dt]).eps / 2 * (1 + 1e-3)


def _case(seed, M, F, K, dt, bias=True):
    x, xf = _g(seed, 1, (M, K), dt)
    w, wf = _g(seed, 2, (2 * F, K), dt, 1.5 / np.sqrt(K))
    b, bf = _g(seed, 3, (2 * F,), "fp32", 0.3) if bias else (None, np.zeros(2 * F))
    return x, xf, w, wf, b, bf


def _check_forward(free, M, F, K, dt, act, bias=True, seed=1):
    x, xf, w, wf, b, bf = _case(seed, M, F, K, dt, bias)
    h, pre = free.op_gated_linear(x, w, b, act=act, want_preact=True)
    ho, zo = ob.gated_linear(xf, wf, bf, act)
    tz = _sum_err(K, dt) * (np.abs(xf) @ np.abs(wf).T + np.abs(bf))
    assert (np.abs(_f64(pre) - zo) <= tz + _half(dt) * np.abs(zo) + TINY).all()
    a, da = ob.gate_act(act, zo[:, :F])
    arg = np.abs(zo[:, :F]) if act == "silu" else np.abs(1.5957691 * (zo[:, :F] + 0.044715 * zo[:, :F] ** 3))
    zu = np.abs(zo[:, F:])
    tol = 1.2 * tz[:, :F] * (zu + tz[:, F:]) + np.abs(a) * tz[:, F:] + (12 + 1.2 * arg) * 2 * U * np.abs(a) * zu
    assert (np.abs(_f64(h) - ho) <= tol + _half(dt) * np.abs(ho) + TINY).all()
    h2 = free.op_gated_linear(x, w, b, act=act)
    assert torch.equal(h, h2) and free.op_device_error() == 0
    return x, w, b


BF16 = [  # M, F, K
    (2, 16, 24), (4, 1000, 2056), (5, 72, 40), (8, 8, 16), (1, 8, 8), (1, 64, 64), (3, 72, 40), (1, 4608, 1152), (2, 1536, 384), (127, 136, 72), (128, 128, 128), (129, 200, 264),
    (255, 64, 1000), (256, 256, 64), (257, 1000, 136), (600, 1536, 384), (1000, 328, 1152), (5000, 136, 200), (77, 40, 4608),
]


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("M,F,K", BF16)
def test_forward_bf16(M, F, K, act):
    import paper_2511_20390_b200 as free
    _check_forward(free, M, F, K, "bf16", act, bias=(M + F) % 3 != 0, seed=M + F + K)


FP32 = [(7, 33, 1001), (9, 40, 260), (32, 17, 64), (1, 1, 1), (1, 5, 3), (2, 64, 64), (33, 65, 31), (100, 130, 257), (129, 64, 16), (64, 256, 64), (500, 96, 384), (1030, 200, 100), (4000, 9, 33)]


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("M,F,K", FP32)
def test_forward_fp32(M, F, K, act):
    import paper_2511_20390_b200 as free
    _check_forward(free, M, F, K, "fp32", act, bias=(M + F) % 3 != 0, seed=M + F + K)


def _check_backward(free, M, F, K, dt, act, seed=1):
    x, xf, w, wf, _, _ = _case(seed, M, F, K, dt)
    pre, zf = _g(seed, 4, (M, 2 * F), dt, 1.3)
    dh, dhf = _g(seed, 5, (M, F), dt, 0.1)
    dx, dw, db = free.op_gated_linear_bwd(x, w, pre, dh, act=act)
    dxo, dwo, dbo = ob.gated_linear_bwd(xf, wf, zf, dhf, act)
    a, da = ob.gate_act(act, zf[:, :F])
    arg = np.abs(zf[:, :F]) if act == "silu" else np.abs(1.5957691 * (zf[:, :F] + 0.044715 * zf[:, :F] ** 3))
    dz = np.concatenate([np.abs(dhf * zf[:, F:] * da), np.abs(dhf * a)], 1)
    # the slope s + g s (1 - s) a' is a sum of terms that can cancel: its error is relative to their sizes
    size = np.concatenate([np.abs(dhf * zf[:, F:]) * (1 + arg * 1.2), np.abs(dhf * zf[:, :F])], 1)
    tz = (16 + 1.2 * np.concatenate([arg, arg], 1)) * 2 * U * size
    step = 2.0 ** -8 if dt == "bf16" else 0.0
    assert (np.abs(_f64(db) - dbo) <= tz.sum(0) + (M + 24) * U * dz.sum(0) + TINY).all()
    err_z = tz + step * (dz + tz)
    tol = err_z @ np.abs(wf) + _sum_err(2 * F, dt) * ((dz + err_z) @ np.abs(wf)) + _half(dt) * np.abs(dxo) + 34 * U * (dz @ np.abs(wf)) + TINY
    assert (np.abs(_f64(dx) - dxo) <= tol).all()
    tol = err_z.T @ np.abs(xf) + _sum_err(M, dt) * ((dz + err_z).T @ np.abs(xf)) + _half(dt) * np.abs(dwo) + 34 * U * (dz.T @ np.abs(xf)) + TINY
    assert (np.abs(_f64(dw) - dwo) <= tol).all()
    if dt == "bf16":
        for got, ref in ((dx, dxo), (dw, dwo)):
            if ref.size >= 4000:
                assert np.linalg.norm(_f64(got) - ref) <= 4e-3 * np.linalg.norm(ref)
    again = free.op_gated_linear_bwd(x, w, pre, dh, act=act)
    assert all(torch.equal(p, q) for p, q in zip((dx, dw, db), again)) and free.op_device_error() == 0
    # each gradient on its own
    assert torch.equal(free.op_gated_linear_bwd(x, w, pre, dh, act=act, want_dw=False, want_dbias=False)[0], dx)
    only = free.op_gated_linear_bwd(x, w, pre, dh, act=act, want_dx=False, want_dbias=False)
    assert only[0] is None and only[2] is None and torch.equal(only[1], dw)
    assert torch.equal(free.op_gated_linear_bwd(x, w, pre, dh, act=act, want_dx=False, want_dw=False)[2], db)


@pytest.mark.parametrize("dt,M,F,K", [
    ("bf16", 64, 216, 8), ("bf16", 65, 224, 136), ("bf16", 130, 136, 72), ("bf16", 257, 64, 8), ("bf16", 1000, 24, 40), ("bf16", 1751, 8, 64), ("bf16", 1750, 8, 64),
    ("fp32", 130, 216, 1146), ("fp32", 600, 64, 1030), ("fp32", 65, 1000, 129), ("fp32", 200, 300, 260), ("fp32", 333, 700, 512),
    ("fp32", 100, 500, 4096), ("fp32", 900, 800, 130), ("fp32", 25, 801, 128), ("fp32", 64, 64, 9001),
    ("fp32", 33, 4849, 5), ("fp32", 35, 216, 1146), ("fp32", 1300, 131, 257), ("fp32", 5000, 33, 31), ("fp32", 700, 250, 64), ("fp32", 20000, 8, 12), ("fp32", 160001, 1, 3),
])
def test_forward_beside_the_choice_of_kernel(dt, M, F, K):
    """Few rows or a narrow layer, just more than that, and contractions that several CTAs share."""
    import paper_2511_20390_b200 as free
    _check_forward(free, M, F, K, dt, "silu", bias=M % 2 == 0, seed=M + F + K)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("M,F,K", BF16 + [(3333, 64, 64), (20, 1536, 384)])
def test_backward_bf16(M, F, K, act):
    import paper_2511_20390_b200 as free
    _check_backward(free, M, F, K, "bf16", act, seed=M + F + K)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("M,F,K", FP32)
def test_backward_fp32(M, F, K, act):
    import paper_2511_20390_b200 as free
    _check_backward(free, M, F, K, "fp32", act, seed=M + F + K)


def test_parts_are_taken_and_reach_every_row():
    # shapes whose products are split along the contraction, and whose row blocks are ragged inside a part
    import paper_2511_20390_b200 as free
    for M, F, K in ((9000, 40, 64), (8193, 136, 72), (300, 2048, 72)):
        _check_backward(free, M, F, K, "bf16", "silu", seed=M)
    _check_backward(free, 6001, 33, 70, "fp32", "gelu", seed=6)


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
def test_extreme_gates(dt):
    # gates far out on both sides: the logistic function saturates without a NaN
    import paper_2511_20390_b200 as free
    M, F, K = 5, 16, 8
    x = torch.zeros(M, K, dtype=DT[dt], device="cuda")
    w = torch.zeros(2 * F, K, dtype=DT[dt], device="cuda")
    vals = torch.tensor([-1e30, -1e4, -200.0, -89.0, -88.0, -60.0, -1.0, 0.0, 1e-30, 1.0, 30.0, 88.0, 89.0, 200.0, 1e4, 1e5], device="cuda")
    b = torch.cat([vals, torch.ones(F, device="cuda")])
    h = free.op_gated_linear(x, w, b, act="silu").double().cpu().numpy()
    v = vals.double().cpu().numpy()
    ref = np.where(v < -700, 0.0, v / (1 + np.exp(np.minimum(-v, 700))))
    assert np.allclose(h, ref, rtol=1e-2 if dt == "bf16" else 1e-4, atol=1e-35)
    g = free.op_gated_linear(x, w, b, act="gelu").double().cpu().numpy()
    assert np.isfinite(g).all() and np.allclose(g[:, -3:], v[-3:], rtol=4e-3) and not g[:, :5].any()
    pre = torch.cat([vals, torch.ones(F, device="cuda")]).to(DT[dt]).repeat(M, 1)
    dx, dw, db = free.op_gated_linear_bwd(x + 1, w, pre, torch.ones(M, F, dtype=DT[dt], device="cuda"), act="silu")
    assert torch.isfinite(dw.float()).all() and torch.isfinite(db).all()
    db = db.cpu().numpy()
    assert np.allclose(db[10:16], M, rtol=1e-6) and not db[:3].any() and np.isclose(db[7], M * 0.5)


def test_a_bad_row_stays_alone():
    import paper_2511_20390_b200 as free
    for dt, K, F in (("bf16", 136, 200), ("fp32", 33, 50)):
        x, _, w, _, b, _ = _case(3, 300, F, K, dt)
        ref = free.op_gated_linear(x, w, b)
        x[17, 3] = float("nan"); x[299, 0] = float("inf")
        got = free.op_gated_linear(x, w, b)
        keep = [i for i in range(300) if i not in (17, 299)]
        assert torch.equal(got[keep], ref[keep]) and torch.isnan(got[17]).all()


def test_empty_batches():
    import paper_2511_20390_b200 as free
    for dt in ("bf16", "fp32"):
        x, w = torch.empty(0, 64, dtype=DT[dt], device="cuda"), torch.ones(2 * 24, 64, dtype=DT[dt], device="cuda")
        h, pre = free.op_gated_linear(x, w, want_preact=True)
        assert h.shape == (0, 24) and pre.shape == (0, 48)
        dx, dw, db = free.op_gated_linear_bwd(x, w, pre, h)
        assert dx.shape == (0, 64) and not dw.any() and not db.any()


def test_what_lies_around_the_outputs_stays():
    import paper_2511_20390_b200 as free
    M, F, K = 130, 72, 40
    x, _, w, _, b, _ = _case(4, M, F, K, "bf16")
    buf = torch.full((2 + M * F + 8 * 130,), 7.0, dtype=torch.bfloat16, device="cuda")
    out = buf[512:512 + M * F].view(M, F)
    ref = free.op_gated_linear(x, w, b)
    free.op_gated_linear(x, w, b, out=out)
    assert torch.equal(out, ref) and (buf[:512] == 7).all() and (buf[512 + M * F:] == 7).all()


def test_streams_and_graphs():
    import paper_2511_20390_b200 as free
    M, F, K = 1500, 384, 264
    x, _, w, _, b, _ = _case(5, M, F, K, "bf16")
    dh, _ = _g(5, 6, (M, F), "bf16", 0.1)
    h, pre = free.op_gated_linear(x, w, b, want_preact=True)
    ref = free.op_gated_linear_bwd(x, w, pre, dh)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = []
    for s in streams:                                              # several at once: every call has its own workspace
        with torch.cuda.stream(s):
            outs.append((free.op_gated_linear(x, w, b),) + free.op_gated_linear_bwd(x, w, pre, dh))
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o[0], h) and all(torch.equal(p, q) for p, q in zip(o[1:], ref))
    graphs = []
    for _ in range(2):                                             # two captured graphs, replayed in turn
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            h2, pre2 = free.op_gated_linear(x, w, b, want_preact=True)
            got = free.op_gated_linear_bwd(x, w, pre2, dh)
        graphs.append((g, h2, got))
    x.mul_(0.5); dh.neg_()
    for g, _, _ in graphs:
        g.replay()
    torch.cuda.synchronize()
    h3, pre3 = free.op_gated_linear(x, w, b, want_preact=True)
    want = free.op_gated_linear_bwd(x, w, pre3, dh)
    for _, h2, got in graphs:
        assert torch.equal(h2, h3) and all(torch.equal(p, q) for p, q in zip(got, want))


def test_first_call_inside_a_capture_is_refused():
    # the error word that the calls share must not be made (and zeroed) inside a graph
    from paper_2511_20390_b200 import binding
    x, w = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(32, 64, dtype=torch.bfloat16, device="cuda")
    kept = dict(binding._ERROR_WORDS)
    binding._ERROR_WORDS.clear()
    refused = False
    try:
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            try:
                binding.op_gated_linear(x, w)
            except RuntimeError:
                refused = True
            x.add_(0.0)                                            # a graph with something in it
    finally:
        binding._ERROR_WORDS.update(kept)
    assert refused
    assert not binding.op_gated_linear(x, w).any()


def test_the_tolerance_sees_swapped_halves():
    # a mistake planted in the definition: gate and up rows exchanged
    x, w = synth.normal(1, 1, (20, 64)).astype(np.float64), synth.normal(1, 2, (32, 64)).astype(np.float64) / 8
    h, _ = ob.gated_linear(x, w)
    swapped, _ = ob.gated_linear(x, np.concatenate([w[16:], w[:16]]))
    assert np.abs(h - swapped).max() > 100 * (64 / 16 + 4) * 4 * U * (np.abs(x) @ np.abs(w).T).max()
