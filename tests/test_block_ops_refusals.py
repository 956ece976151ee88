"""What the block operators refuse, at the C boundary and in the binding.  Every call here ends on the host (no GPU needed):
the pointers are never dereferenced."""
import ctypes as C

import pytest
import torch

P, ODD = C.c_void_p(4096), C.c_void_p(4100)
ARG, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE = -1, -2, -3, -4, -6


@pytest.fixture(scope="module")
def L():
    from paper_2511_20390_b200.build import build
    build()
    from paper_2511_20390_b200 import binding
    return binding.lib()


def _norm(L, xd=0, yd=1, g=2, rows=3, D=64, x=P, xs=64, w=P, b=P, ms=64, unit=0, eps=1e-6, y=P, ys=64, st=P):
    return L.free_op_layer_norm(xd, yd, g, rows, D, x, xs, w, b, ms, unit, eps, y, ys, st, None)


def _norm_bwd(L, xd=0, yd=1, g=2, rows=3, D=64, x=P, xs=64, dy=P, dys=64, st=P, w=P, ms=64, unit=0, res=None, rs=0, dx=P, dxs=64,
              dw=P, db=P, dms=64, ws=None, need=0):
    return L.free_op_layer_norm_bwd(xd, yd, g, rows, D, x, xs, dy, dys, st, w, ms, unit, res, rs, dx, dxs, dw, db, dms, ws, need, None)


def test_layer_norm(L):
    assert _norm(L, xd=2) == ARG and _norm(L, yd=-1) == ARG
    assert _norm(L, eps=-1e-6) == ARG and _norm(L, eps=float("nan")) == ARG
    assert _norm(L, x=None) == ARG and _norm(L, y=None) == ARG
    assert _norm(L, D=0) == SHAPE and _norm(L, g=-1) == SHAPE and _norm(L, rows=-1) == SHAPE
    assert _norm(L, xs=63) == SHAPE and _norm(L, ys=63) == SHAPE and _norm(L, ms=-64) == SHAPE
    assert _norm(L, x=ODD) == ALIGN and _norm(L, y=ODD) == ALIGN and _norm(L, w=C.c_void_p(4098)) == ALIGN
    assert _norm(L, D=8193, xs=8193, ys=8193) == UNSUPPORTED
    assert _norm(L, rows=0, x=None, y=None) == 0 and _norm(L, g=0, x=None, y=None) == 0


def test_layer_norm_bwd(L):
    assert _norm_bwd(L, xd=2) == ARG and _norm_bwd(L, yd=5) == ARG
    for k in ("x", "dy", "st", "dx"):
        assert _norm_bwd(L, **{k: None}) == ARG
    assert _norm_bwd(L, D=0) == SHAPE and _norm_bwd(L, rows=-2) == SHAPE
    for k in ("xs", "dys", "dxs", "dms"):
        assert _norm_bwd(L, **{k: 63}) == SHAPE
    assert _norm_bwd(L, res=P, rs=63) == SHAPE
    for k in ("x", "dy", "dx"):
        assert _norm_bwd(L, **{k: ODD}) == ALIGN
    assert _norm_bwd(L, res=ODD, rs=64) == ALIGN and _norm_bwd(L, dw=C.c_void_p(4098)) == ALIGN
    big = dict(D=8193, xs=8193, dys=8193, dxs=8193, dms=8193)
    assert _norm_bwd(L, **big) == UNSUPPORTED
    need = L.free_op_layer_norm_bwd_workspace_bytes(2, 1000, 1152)
    wide = dict(rows=1000, D=1152, xs=1152, dys=1152, dxs=1152, dms=1152)
    assert need > 0 and need % 4 == 0
    assert _norm_bwd(L, **wide) == WORKSPACE and _norm_bwd(L, ws=P, need=need - 1, **wide) == WORKSPACE
    assert _norm_bwd(L, g=0, x=None, dy=None, st=None, dx=None) == 0
    assert L.free_op_layer_norm_bwd_workspace_bytes(0, 10, 64) == 0 and L.free_op_layer_norm_bwd_workspace_bytes(1, 1, 64) == 0
    # the workspace grows with what it holds and stays small beside the rows
    for g, r, D in ((1, 24576, 1152), (24, 1024, 1152), (1, 100000, 64), (3, 5000, 8192)):
        assert L.free_op_layer_norm_bwd_workspace_bytes(g, r, D) <= g * r * D * 4 / 4


def _rope(L, dt=0, pairing=0, freq=0, inv=0, n=2, t=3, h=4, d=64, axes=(32, 32), base=1e4, pos=P, ps=0, x=P, xs=(768, 256, 64),
          y=P, ys=(768, 256, 64), no_axes=False):
    arr = None if no_axes else (C.c_int32 * max(1, len(axes)))(*axes)
    return L.free_op_rope_axes(dt, pairing, freq, inv, n, t, h, d, len(axes), arr, base, pos, ps, x, *xs, y, *ys, None)


def test_rope(L):
    assert _rope(L, dt=2) == ARG and _rope(L, pairing=2) == ARG and _rope(L, freq=-1) == ARG and _rope(L, no_axes=True) == ARG
    assert _rope(L, base=0.0) == ARG and _rope(L, base=float("inf")) == ARG and _rope(L, base=float("nan")) == ARG
    assert _rope(L, pos=None) == ARG and _rope(L, x=None) == ARG and _rope(L, y=None) == ARG
    assert _rope(L, axes=()) == SHAPE and _rope(L, axes=(8,) * 5) == SHAPE
    assert _rope(L, axes=(31, 33)) == SHAPE and _rope(L, axes=(-2, 4)) == SHAPE and _rope(L, axes=(0, 0)) == SHAPE
    assert _rope(L, axes=(64, 2)) == SHAPE and _rope(L, n=-1) == SHAPE and _rope(L, h=0) == SHAPE
    assert _rope(L, xs=(768, -256, 64)) == SHAPE and _rope(L, ps=-1) == SHAPE
    assert _rope(L, ys=(768, 256, 32)) == SHAPE and _rope(L, ys=(768, 0, 64)) == SHAPE       # outputs on one another
    assert _rope(L, d=63, axes=(32,), xs=(1000, 300, 63), ys=(1000, 300, 63)) == UNSUPPORTED
    assert _rope(L, d=512, axes=(258,), xs=(9000, 3000, 512), ys=(9000, 3000, 512)) == UNSUPPORTED
    assert _rope(L, x=C.c_void_p(4098)) == ALIGN and _rope(L, dt=1, y=C.c_void_p(4097)) == ALIGN
    assert _rope(L, n=0, pos=None, x=None, y=None) == 0 and _rope(L, t=0, pos=None, x=None, y=None) == 0


def test_binding_checks(L):
    import paper_2511_20390_b200 as free
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        free.op_layer_norm(x)                                      # not on a GPU
    with pytest.raises(ValueError):
        free.op_layer_norm(torch.zeros(2, 3, 4))
    with pytest.raises(ValueError):
        free.op_layer_norm(x, rows_per_group=3)                    # not whole groups
    with pytest.raises(ValueError):
        free.op_rope_axes(torch.zeros(2, 3, 4), torch.zeros(3, 1), (4,))
    with pytest.raises(ValueError):
        free.op_rope_axes(torch.zeros(1, 3, 2, 4), torch.zeros(3, 1), (4,), pairing="thirds")


def _gated(L, dt=1, act=0, M=4, F=64, K=64, x=P, w=P, b=P, h=P, pre=P, err=P):
    return L.free_op_gated_linear(dt, act, M, F, K, x, w, b, h, pre, err, None)


def _gated_bwd(L, dt=1, act=0, M=4, F=64, K=64, x=P, w=P, pre=P, dh=P, dx=P, dw=P, db=P, ws=None, need=0, err=P):
    return L.free_op_gated_linear_bwd(dt, act, M, F, K, x, w, pre, dh, dx, dw, db, ws, need, err, None)


def test_gated_linear(L):
    assert _gated(L, dt=2) == ARG and _gated(L, act=2) == ARG and _gated(L, act=-1) == ARG
    for k in ("x", "w", "h", "err"):
        assert _gated(L, **{k: None}) == ARG
    assert _gated(L, M=-1) == SHAPE and _gated(L, F=0) == SHAPE and _gated(L, K=0) == SHAPE
    for k in ("x", "w", "h", "pre"):
        assert _gated(L, **{k: ODD}) == ALIGN
    assert _gated(L, b=C.c_void_p(4098)) == ALIGN
    assert _gated(L, F=60) == UNSUPPORTED and _gated(L, K=36) == UNSUPPORTED        # rows that are not multiples of 16 bytes
    assert _gated(L, M=(1 << 30) + 1) == UNSUPPORTED and _gated(L, F=(1 << 28) + 8) == UNSUPPORTED and _gated(L, K=1 << 30) == UNSUPPORTED
    assert _gated(L, M=0, x=None, w=None, h=None, err=None) == 0


def test_gated_linear_bwd(L):
    assert _gated_bwd(L, dt=3) == ARG and _gated_bwd(L, act=7) == ARG
    for k in ("x", "w", "pre", "dh", "err"):
        assert _gated_bwd(L, **{k: None}) == ARG
    assert _gated_bwd(L, M=-1) == SHAPE and _gated_bwd(L, F=0) == SHAPE
    for k in ("x", "w", "pre", "dh", "dx", "dw"):
        assert _gated_bwd(L, **{k: ODD}) == ALIGN
    assert _gated_bwd(L, F=60) == UNSUPPORTED and _gated_bwd(L, K=36) == UNSUPPORTED
    assert _gated_bwd(L, M=(1 << 30) + 1) == UNSUPPORTED and L.free_op_gated_linear_bwd_workspace_bytes(1, 4, 1 << 29, 64) == 0
    need = L.free_op_gated_linear_bwd_workspace_bytes(1, 4, 64, 64)
    assert need >= 4 * 128 * 2
    assert _gated_bwd(L) == WORKSPACE and _gated_bwd(L, ws=P, need=need - 1) == WORKSPACE
    assert _gated_bwd(L, dx=None, dw=None, db=None) == 0
    assert L.free_op_gated_linear_bwd_workspace_bytes(1, 4, 60, 64) == 0 and L.free_op_gated_linear_bwd_workspace_bytes(0, 0, 60, 64) == 0
    # dz and, where a product is split, its parts: bounded by a few times the operands
    for dt, M, F, K in ((1, 24576, 4608, 1152), (1, 1, 4608, 1152), (1, 9000, 40, 64), (0, 6001, 33, 70), (0, 1, 1, 1)):
        n = L.free_op_gated_linear_bwd_workspace_bytes(dt, M, F, K)
        assert n >= M * 2 * F * (2 if dt else 4)
        assert n <= M * 2 * F * 4 + 1200 * 2 * F * 4 + 64 * 4 * K * (max(M, 2 * F) + 256) + 1024


def test_gated_binding_checks(L):
    import paper_2511_20390_b200 as free
    x, w = torch.zeros(4, 8), torch.zeros(16, 8)
    for call in (lambda: free.op_gated_linear(x, w), lambda: free.op_gated_linear(x, torch.zeros(15, 8)),
                 lambda: free.op_gated_linear(x, w, act="relu"), lambda: free.op_gated_linear(torch.zeros(4, 2, 4), w),
                 lambda: free.op_gated_linear_bwd(x, w, torch.zeros(4, 16), torch.zeros(4, 8), act="tanh")):
        with pytest.raises(ValueError):
            call()
    assert free.op_device_error("cuda:0") == 0                      # nothing has run there
