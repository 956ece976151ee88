"""free_op_rope_axes against the fp64 definition.

Tolerance (u = 2^-24): the angle's remainder is rounded once to fp32 (at most u of half a turn: pi u), sine and cosine are good
to 2 units, two products and a sum: (|a| + |b|) 8 u in all; then half a step of the output's type."""
import numpy as np
import pytest
import torch

import synth
from oracle import block_ops as ob

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _x(seed, shape, dt):
    return torch.from_numpy(synth.normal(seed, 1, shape)).to(DT[dt]).cuda()


def _check(got, x, pos, axes, dt, **kw):
    xf = x.double().cpu().numpy()
    ref = ob.rope_axes(xf, pos.double().cpu().numpy(), axes, **kw)
    P, R = sum(axes) // 2, sum(axes)
    size = np.zeros_like(xf)
    if kw.get("pairing", "interleaved") == "interleaved":
        s = np.abs(xf[..., 0:R:2]) + np.abs(xf[..., 1:R:2])
        size[..., 0:R:2] = s; size[..., 1:R:2] = s
    else:
        s = np.abs(xf[..., :P]) + np.abs(xf[..., P:R])
        size[..., :P] = s; size[..., P:R] = s
    half = torch.finfo(DT[dt]).eps / 2
    tol = 8 * U * size + half * np.abs(ref) * (size > 0) * (1 + 1e-3)
    err = np.abs(got.double().cpu().numpy() - ref)
    assert (err <= tol).all(), (err - tol).max()


CASES = [  # n_seq, n_tok, heads, d_head, axes
    (1, 1, 1, 2, (2,)), (1, 3, 1, 4, (2,)), (2, 5, 3, 6, (2, 2, 2)), (1, 1, 16, 72, (36, 36)), (3, 64, 16, 72, (36, 36)),
    (2, 30, 12, 72, (24, 24, 24)), (1, 257, 6, 64, (32, 32)), (2, 33, 2, 80, (40, 20)), (1, 100, 24, 128, (16, 56, 56)),
    (1, 9, 3, 128, (128,)), (1, 7, 2, 256, (64, 64, 64, 64)), (2, 11, 1, 16, (0, 16)), (1, 19, 70, 64, (20, 22)),
    (1, 5, 5, 34, (34,)), (4, 1, 300, 8, (8,)), (1, 1000, 1, 2, (2,)),
]


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("pairing", ["interleaved", "halves"])
@pytest.mark.parametrize("case", CASES)
def test_matches_the_definition(case, pairing, dt):
    import paper_2511_20390_b200 as free
    n, t, h, d, axes = case
    x = _x(n + t + d, (n, t, h, d), dt)
    pos = torch.from_numpy(np.stack([np.arange(t) % (5 + 3 * a) for a in range(len(axes))], 1).astype(np.float32)).cuda()
    for joint in (False, True):
        y = free.op_rope_axes(x, pos, axes, pairing=pairing, joint_freq=joint)
        _check(y, x, pos, axes, dt, pairing=pairing, joint_freq=joint)
        _check(free.op_rope_axes(x, pos, axes, pairing=pairing, joint_freq=joint, inverse=True), x, pos, axes, dt, pairing=pairing,
               joint_freq=joint, inverse=True)


@pytest.mark.parametrize("pairing", ["interleaved", "halves"])
def test_far_fractional_and_negative_positions(pairing):
    import paper_2511_20390_b200 as free
    x = _x(1, (2, 6, 4, 72), "fp32")
    p = np.array([[0, 0], [16777216, 1], [-100000, 0.25], [1048576, -3.5], [5e6, 4e6], [1, 1e7]], np.float32)
    pos = torch.from_numpy(np.stack([p, p[::-1] * 0.5])).cuda()                       # another set for each sequence
    for base in (10000.0, 500.0, 1.0e6):
        _check(free.op_rope_axes(x, pos, (36, 36), base=base, pairing=pairing), x, pos, (36, 36), "fp32", base=base, pairing=pairing)


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("pairing", ["interleaved", "halves"])
@pytest.mark.parametrize("heads,d", [(16, 72), (3, 18), (2, 34)])
def test_inside_the_packed_projection(heads, d, pairing, dt):
    import paper_2511_20390_b200 as free
    n, t, axes = 2, 37, (d // 4 * 2, d - d // 4 * 2) if d % 4 == 0 else (d - 8, 8)
    qkv = _x(4, (n, t, 3 * heads, d), dt)
    pos = torch.from_numpy(np.stack([np.arange(t) // 6, np.arange(t) % 6], 1).astype(np.float32)).cuda()
    before = qkv.clone()
    y = free.op_rope_axes(qkv[:, :, :2 * heads], pos, axes, pairing=pairing)
    assert torch.equal(qkv, before) and y.is_contiguous()
    _check(y, before[:, :, :2 * heads], pos, axes, dt, pairing=pairing)
    k = free.op_rope_axes(qkv[:, :, heads:2 * heads], pos, axes, pairing=pairing)     # starts at any element
    assert torch.equal(k, y[:, :, heads:])
    got = free.op_rope_axes(qkv[:, :, :2 * heads], pos, axes, pairing=pairing, out=qkv[:, :, :2 * heads])     # in place
    assert torch.equal(got, y) and torch.equal(qkv[:, :, 2 * heads:], before[:, :, 2 * heads:])
    # heads in front of the tokens: another order of strides
    z = before[:, :, :2 * heads].transpose(1, 2).contiguous().transpose(1, 2)
    assert torch.equal(free.op_rope_axes(z, pos, axes, pairing=pairing), y)
    out = torch.zeros(n, 2 * heads, t, d, dtype=DT[dt], device="cuda").transpose(1, 2)
    assert torch.equal(free.op_rope_axes(z, pos, axes, pairing=pairing, out=out), y)


def test_copied_elements_keep_their_bits():
    import paper_2511_20390_b200 as free
    for pairing in ("interleaved", "halves"):
        for dt in ("bf16", "fp32"):
            x = _x(6, (1, 20, 3, 64), dt)
            x[..., 36:] = float("inf")
            x[..., 40] = float("nan")
            x[..., 41] = -0.0
            pos = torch.arange(20, dtype=torch.float32, device="cuda")[:, None]
            y = free.op_rope_axes(x, pos, (36,), pairing=pairing)
            kind = torch.int16 if dt == "bf16" else torch.int32
            assert torch.equal(y[..., 36:].contiguous().view(kind), x[..., 36:].contiguous().view(kind))
            assert torch.isfinite(y[..., :36]).all()


def test_empty_streams_and_graphs():
    import paper_2511_20390_b200 as free
    assert free.op_rope_axes(torch.empty(0, 5, 2, 8, device="cuda"), torch.zeros(5, 1, device="cuda"), (8,)).shape == (0, 5, 2, 8)
    assert free.op_rope_axes(torch.empty(2, 0, 2, 8, device="cuda"), torch.zeros(0, 1, device="cuda"), (8,)).shape == (2, 0, 2, 8)
    x = _x(8, (2, 300, 6, 64), "bf16")
    pos = torch.arange(300, dtype=torch.float32, device="cuda")[:, None].repeat(1, 2)
    ref = free.op_rope_axes(x, pos, (32, 32))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = free.op_rope_axes(x, pos, (32, 32))
    side.synchronize()
    assert torch.equal(got, ref)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = free.op_rope_axes(x, pos, (32, 32))
    x.neg_(); pos.add_(1.0)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, free.op_rope_axes(x, pos, (32, 32)))


def test_offsets_past_32_bits():
    import paper_2511_20390_b200 as free
    # two tokens more than 2^32 elements apart in one allocation (bf16: 8.6 GB)
    step = (1 << 32) + 64
    buf = torch.zeros(step + 128, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((1, 2, 2, 64), (0, step, 64, 1))
    x.copy_(_x(11, (1, 2, 2, 64), "bf16"))
    pos = torch.tensor([[3.0], [7.0]], device="cuda")
    want = free.op_rope_axes(x.contiguous(), pos, (64,))
    assert torch.equal(free.op_rope_axes(x, pos, (64,)), want)
    free.op_rope_axes(x, pos, (64,), out=x)
    assert torch.equal(x, want)
