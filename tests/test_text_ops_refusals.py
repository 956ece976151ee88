"""What the attention to an encoder's states and the RMS norm refuse, at the C boundary and in the binding.  Every call here ends on
the host (no GPU needed): the pointers are never dereferenced."""
import ctypes as C
import re
from pathlib import Path

import pytest
import torch

P, ODD = 4096, 4098                                                # aligned; 2 bytes off
ARG, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE = -1, -2, -3, -4, -6


@pytest.fixture(scope="module")
def L():
    from paper_2511_20390_b200.build import build
    build()
    from paper_2511_20390_b200 import binding
    return binding.lib()


class Shape(C.Structure):
    """free_cross_attn as a C compiler lays it out."""
    _fields_ = ([(n, C.c_void_p) for n in ("q", "k", "v")] +
                [(f"{m}_{s}", C.c_int64) for m in "qkv" for s in ("seq", "tok", "head")] +
                [(n, C.c_void_p) for n in ("kv_lens", "kv_offsets", "kv_seq", "kv_mask")] +
                [(n, C.c_int32) for n in ("dtype", "n_seq", "n_q", "heads", "kv_heads", "d_head", "n_enc", "n_kv", "kv_rows")] + [("scale", C.c_float)])


def _shape(**kw):
    v = dict(q=P, k=P, v=P, q_seq=640, q_tok=128, q_head=64, k_seq=1280, k_tok=128, k_head=64, v_seq=1280, v_tok=128, v_head=64, kv_lens=0, kv_offsets=0,
             kv_seq=0, kv_mask=0, dtype=1, n_seq=2, n_q=5, heads=2, kv_heads=2, d_head=64, n_enc=2, n_kv=10, kv_rows=10, scale=0.125)
    v.update(kw)
    return v


def _pack(**kw):
    return bytes(Shape(**_shape(**kw)))


def _fwd(L, out=P, os=(640, 128, 64), lse=P, ws=None, need=0, err=P, **kw):
    return L.free_op_cross_attention(_pack(**kw), out, *os, lse, ws, need, err, None)


def _bwd(L, out=P, os=(640, 128, 64), lse=P, g=P, gs=(640, 128, 64), dq=P, dqs=(640, 128, 64), dk=P, dks=(1280, 128, 64), dv=P, dvs=(1280, 128, 64), ws=P,
         need=1 << 40, err=P, **kw):
    return L.free_op_cross_attention_bwd(_pack(**kw), out, *os, lse, g, *gs, dq, *dqs, dk, *dks, dv, *dvs, ws, need, err, None)


def test_the_binding_packs_the_struct_as_c_lays_it_out(L):
    from paper_2511_20390_b200 import binding
    v = {n: i + 1 for i, (n, _) in enumerate(Shape._fields_)}
    assert binding._CROSS.size == C.sizeof(Shape)
    assert binding._CROSS.pack(*v.values()) == bytes(Shape(**v))
    # and in the order of the header
    head = (Path(binding.__file__).resolve().parents[1] / "include" / "free_b200.h").read_text()
    body = re.search(r"typedef struct free_cross_attn \{(.*?)\} free_cross_attn;", head, re.S).group(1)
    names = [n for line in body.split(";") for n in re.findall(r"\*?\s*(\w+)\s*(?:,|$)", re.sub(r"^\s*(const\s+)?\w+\s*", "", line.strip()))]
    assert names == [n for n, _ in Shape._fields_]


def _common(f):
    assert f(dtype=2) == ARG and f(dtype=-1) == ARG
    for s in (0.0, -1.0, float("nan"), float("inf")):
        assert f(scale=s) == ARG
    assert f(kv_lens=P, kv_offsets=P) == ARG
    assert f(q=0) == ARG and f(k=0) == ARG and f(v=0) == ARG and f(err=None) == ARG
    for n in ("n_seq", "n_q", "n_enc", "n_kv", "kv_rows"):
        assert f(**{n: -1}) == SHAPE
    assert f(heads=0) == SHAPE and f(kv_heads=0) == SHAPE and f(d_head=0) == SHAPE
    assert f(heads=3) == SHAPE                                     # not a multiple of the key heads
    assert f(n_seq=3) == SHAPE and f(n_enc=0) == SHAPE             # sequences that share no whole number of states
    for n in ("q_seq", "q_tok", "q_head", "k_seq", "k_tok", "k_head", "v_seq", "v_tok", "v_head"):
        assert f(**{n: -64}) == SHAPE
    assert f(d_head=129) == UNSUPPORTED
    assert f(n_seq=1 << 30, n_enc=1 << 30) == UNSUPPORTED and f(kv_seq=P, n_enc=1 << 30, kv_heads=2, n_kv=100) == UNSUPPORTED
    for n in ("q", "k", "v"):
        assert f(**{n: 4097}) == ALIGN and f(dtype=0, **{n: ODD}) == ALIGN
    for n in ("kv_lens", "kv_offsets", "kv_seq"):
        assert f(**{n: ODD}) == ALIGN


def test_cross_attention(L):
    _common(lambda **kw: _fwd(L, **kw))
    assert _fwd(L, out=None) == ARG and _fwd(L, out=4097) == ALIGN and _fwd(L, lse=ODD) == ALIGN
    for os in ((-640, 128, 64), (640, 128, 32), (640, 64, 64), (0, 128, 64), (640, 0, 64), (639, 128, 64)):      # rows on one another
        assert _fwd(L, os=os) == SHAPE
    assert _fwd(L, n_seq=0, q=0, k=0, v=0, out=None, err=None) == 0 and _fwd(L, n_q=0, q=0, out=None) == 0
    # few tokens over many states are split, and the parts need a workspace
    long = dict(n_seq=1, n_enc=1, n_q=1, n_kv=100000, q_seq=128, k_seq=12800000, v_seq=12800000)
    need = L.free_op_cross_attention_workspace_bytes(_pack(**long))
    assert need > 0
    assert _fwd(L, **long) == WORKSPACE and _fwd(L, ws=P, need=need - 1, **long) == WORKSPACE and _fwd(L, ws=P + 8, need=need, **long) == ALIGN
    assert L.free_op_cross_attention_workspace_bytes(_pack()) == 0
    assert L.free_op_cross_attention_workspace_bytes(_pack(d_head=129)) == 0 and L.free_op_cross_attention_workspace_bytes(None) == 0
    assert L.free_op_cross_attention(None, P, 640, 128, 64, P, None, 0, P, None) == ARG


def test_cross_attention_bwd(L):
    _common(lambda **kw: _bwd(L, **kw))
    assert _bwd(L, out=None) == ARG and _bwd(L, lse=None) == ARG and _bwd(L, g=None) == ARG
    assert _bwd(L, dk=None) == ARG and _bwd(L, dv=None) == ARG     # both or neither
    assert _bwd(L, out=4097) == ALIGN and _bwd(L, g=4097) == ALIGN and _bwd(L, dq=4097) == ALIGN and _bwd(L, dk=4097) == ALIGN and _bwd(L, lse=ODD) == ALIGN
    assert _bwd(L, os=(-1, 128, 64)) == SHAPE and _bwd(L, gs=(640, -1, 64)) == SHAPE
    assert _bwd(L, dqs=(640, 0, 64)) == SHAPE and _bwd(L, dks=(0, 128, 64)) == SHAPE and _bwd(L, dvs=(1280, 128, 32)) == SHAPE
    need = L.free_op_cross_attention_bwd_workspace_bytes(_pack())
    assert need >= 2 * 5 * 2 * 4
    assert _bwd(L, ws=None) == WORKSPACE and _bwd(L, need=need - 1) == WORKSPACE and _bwd(L, ws=P + 8) == ALIGN
    # parts of dk and dv stay small beside states of which few are named
    for dt in (0, 1):
        for rows, n_kv, d in ((1 << 20, 64, 64), (100, 100, 128), (3000, 3000, 40), (1 << 24, 1, 8)):
            n = L.free_op_cross_attention_bwd_workspace_bytes(_pack(dtype=dt, n_seq=1, n_enc=1, n_q=4096, kv_offsets=P, kv_rows=rows, n_kv=n_kv, d_head=d, kv_heads=1))
            assert 0 < n <= (64 << 20) + 1024 + 2 * 4096 * 4
    # and items of millions of tiles are split whatever the blocks of states
    many = dict(n_seq=1 << 20, n_enc=1, n_q=128, heads=1, kv_heads=1, n_kv=20000, kv_rows=20000, q_seq=128 * 64, q_tok=64, k_seq=20000 * 64, v_seq=20000 * 64)
    rows = (1 << 20) * 128 * 4
    assert L.free_op_cross_attention_bwd_workspace_bytes(_pack(**many)) >= rows + 2 * 2 * 20000 * 64 * 4
    assert L.free_op_cross_attention_bwd_workspace_bytes(_pack(**{**many, "n_seq": 1 << 12})) < (1 << 12) * 128 * 4 + 1024
    # nothing to be written: no gradient wanted, or no token and no state
    assert _bwd(L, n_seq=0, n_enc=0, q=0, k=0, v=0, out=None, lse=None, g=None, dq=None, ws=None, err=None) == 0
    assert _bwd(L, n_q=0, n_kv=0, out=None, lse=None, g=None, dq=None, ws=None, err=None) == 0
    # without tokens the states' gradients are zeros, and their inputs are looked at all the same
    none = dict(n_seq=0, q=0, out=None, lse=None, g=None, dq=None, ws=None, err=None)
    assert _bwd(L, k=0, **none) == ARG and _bwd(L, v=0, **none) == ARG and _bwd(L, kv_lens=ODD, **none) == ALIGN and _bwd(L, k=4097, **none) == ALIGN
    assert L.free_op_cross_attention_bwd_workspace_bytes(_pack(kv_heads=0)) == 0


def _rms(L, xd=1, rd=0, yd=1, g=2, rows=3, H=1, D=64, x=P, xt=64, xh=0, res=None, rs=64, h=None, hs=64, w=P, ms=64, unit=0, eps=1e-6, y=P, yt=64, yh=0,
         sc=None, ss=1, block=0, rstd=P):
    return L.free_op_rms_norm(xd, rd, yd, g, rows, H, D, x, xt, xh, res, rs, h, hs, w, ms, unit, eps, y, yt, yh, sc, ss, block, rstd, None)


def test_rms_norm(L):
    assert _rms(L, xd=2) == ARG and _rms(L, yd=3) == ARG and _rms(L, yd=-1) == ARG and _rms(L, res=P, rd=2) == ARG
    assert _rms(L, eps=-1.0) == ARG and _rms(L, eps=float("nan")) == ARG
    assert _rms(L, x=None) == ARG and _rms(L, y=None) == ARG and _rms(L, h=P) == ARG                   # a sum without a residual
    assert _rms(L, g=-1) == SHAPE and _rms(L, rows=-1) == SHAPE and _rms(L, D=0) == SHAPE and _rms(L, H=0) == SHAPE and _rms(L, H=4) == SHAPE
    assert _rms(L, xt=-64) == SHAPE and _rms(L, yt=63) == SHAPE and _rms(L, ms=-64) == SHAPE
    assert _rms(L, res=P, rs=63) == SHAPE and _rms(L, res=P, h=P, hs=63) == SHAPE
    heads = dict(H=3, rows=6, xt=192, xh=64, yt=192, yh=64)
    assert _rms(L, yt=191, **{k: v for k, v in heads.items() if k != "yt"}) == SHAPE and _rms(L, yh=63, **{k: v for k, v in heads.items() if k != "yh"}) == SHAPE
    assert _rms(L, res=P, **heads) == ARG and _rms(L, yd=2, sc=P, **heads) == ARG                       # of rows only
    assert _rms(L, yd=2) == ARG and _rms(L, yd=2, sc=P, block=64) == ARG and _rms(L, yd=2, sc=P, ss=0) == SHAPE
    assert _rms(L, yd=2, sc=P, block=128, D=200, xt=200, yt=200, ss=1) == SHAPE
    assert _rms(L, x=4097) == ALIGN and _rms(L, xd=0, x=ODD) == ALIGN and _rms(L, y=4097) == ALIGN and _rms(L, res=ODD) == ALIGN
    assert _rms(L, w=ODD) == ALIGN and _rms(L, rstd=ODD) == ALIGN and _rms(L, yd=2, sc=ODD) == ALIGN
    assert _rms(L, D=8193, xt=8193, yt=8193) == UNSUPPORTED
    assert _rms(L, g=0, x=None, y=None) == 0 and _rms(L, rows=0, x=None, y=None) == 0


def _rms_bwd(L, xd=1, yd=1, g=2, rows=3, H=1, D=64, h=P, ht=64, hh=0, dy=P, dyt=64, dyh=0, rstd=P, w=P, ms=64, unit=0, res=None, rt=0, rh=0, dx=P, dxt=64, dxh=0,
             dw=P, dms=64, ws=None, need=0):
    return L.free_op_rms_norm_bwd(xd, yd, g, rows, H, D, h, ht, hh, dy, dyt, dyh, rstd, w, ms, unit, res, rt, rh, dx, dxt, dxh, dw, dms, ws, need, None)


def test_rms_norm_bwd(L):
    assert _rms_bwd(L, xd=2) == ARG and _rms_bwd(L, yd=2) == ARG
    for k in ("h", "dy", "rstd", "dx"):
        assert _rms_bwd(L, **{k: None}) == ARG
    assert _rms_bwd(L, D=0) == SHAPE and _rms_bwd(L, rows=-2) == SHAPE and _rms_bwd(L, H=5) == SHAPE
    for k in ("ht", "dyt", "dxt", "dms"):
        assert _rms_bwd(L, **{k: -1}) == SHAPE
    assert _rms_bwd(L, dxt=63) == SHAPE and _rms_bwd(L, dms=63) == SHAPE and _rms_bwd(L, res=P, rt=-1) == SHAPE
    for k in ("h", "dy", "dx"):
        assert _rms_bwd(L, **{k: 4097}) == ALIGN
    for k in ("rstd", "w", "dw"):
        assert _rms_bwd(L, **{k: ODD}) == ALIGN
    assert _rms_bwd(L, D=8193, ht=8193, dyt=8193, dxt=8193, dms=8193) == UNSUPPORTED
    # heads wider than a lane group's registers have to lie evenly apart
    wide = dict(H=2, rows=4, D=600, ht=1300, hh=600, dyt=1200, dyh=600, dxt=1200, dxh=600, dms=600)
    assert _rms_bwd(L, **wide) == UNSUPPORTED
    need = L.free_op_rms_norm_bwd_workspace_bytes(2, 1000, 1152)
    many = dict(rows=1000, D=1152, ht=1152, dyt=1152, dxt=1152, dms=1152)
    assert need > 0 and _rms_bwd(L, **many) == WORKSPACE and _rms_bwd(L, ws=P, need=need - 1, **many) == WORKSPACE
    assert _rms_bwd(L, g=0, h=None, dy=None, rstd=None, dx=None) == 0
    assert L.free_op_rms_norm_bwd_workspace_bytes(0, 10, 64) == 0 and L.free_op_rms_norm_bwd_workspace_bytes(1, 10, 8193) == 0


def test_binding(L):
    import paper_2511_20390_b200 as free
    x = torch.zeros(4, 8)
    q, k = torch.zeros(2, 3, 4, 8), torch.zeros(2, 5, 2, 8)
    i32 = torch.zeros(3, dtype=torch.int32)
    for call in (
            lambda: free.op_rms_norm(x),                           # not on a GPU
            lambda: free.op_rms_norm(torch.zeros(8)), lambda: free.op_rms_norm(x, rows_per_group=3), lambda: free.op_rms_norm(torch.zeros(4, 8, dtype=torch.float64)),
            lambda: free.op_rms_norm_bwd(torch.zeros(8), x, torch.zeros(4)), lambda: free.op_rms_norm_bwd(x, x, torch.zeros(4)),
            lambda: free.op_cross_attention(q, k, k), lambda: free.op_cross_attention(x, k, k), lambda: free.op_cross_attention(q, x, x),
            lambda: free.op_cross_attention(q, k, k[:, :4]), lambda: free.op_cross_attention(q, k.bfloat16(), k), lambda: free.op_cross_attention(q, k[..., :4], k[..., :4]),
            lambda: free.op_cross_attention(q.transpose(2, 3), k, k), lambda: free.op_cross_attention(q, k, k, kv_offsets=i32),
            lambda: free.op_cross_attention_bwd(q, k, k, q, torch.zeros(2, 4, 3), q)):
        with pytest.raises(ValueError):
            call()
