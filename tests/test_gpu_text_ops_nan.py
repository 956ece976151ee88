"""NaN that counts in the attention to an encoder's states: a query or a state that holds one gives NaN, in out, lse and gradients,
however the states are split; everything that it does not reach is as without it.

Finite rows are held against fp64.  With u = 2^-24 and E = (d + 8) u scale sum |q k| + 8 u, the error of e^S, out is off by at most
sum p |v| (2 E + (n + 16) u [+ 2^-8: probabilities in bf16]) and half a step of its type, lse by E + (n + 16) u + 4 u |lse|."""
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF, FP = torch.bfloat16, torch.float32

# (dtype, n_seq, n_enc, n_q, n_kv, heads, kv_heads, d): few rows, whole and split; tensor cores, whole and split; CUDA cores
SHAPES = [(BF, 2, 2, 1, 77, 4, 2, 64), (BF, 2, 2, 1, 5000, 8, 2, 128), (FP, 2, 1, 2, 3000, 2, 2, 40), (BF, 4, 2, 150, 200, 4, 2, 72),
          (BF, 2, 2, 20, 4200, 2, 2, 64), (BF, 2, 2, 30, 100, 2, 1, 36), (FP, 2, 2, 70, 150, 4, 2, 64)]


def _inputs(shape, seed=1):
    dt, n_seq, n_enc, n_q, n_kv, heads, kvh, d = shape
    gen = torch.Generator("cuda").manual_seed(seed)
    mk = lambda *s: torch.randn(*s, device="cuda", generator=gen).to(dt)
    return mk(n_seq, n_q, heads, d), mk(n_enc, n_kv, kvh, d), mk(n_enc, n_kv, kvh, d), mk(n_seq, n_q, heads, d)


def _agrees(out, lse, q, k, v):
    """Finite results against fp64; both of them NaN where fp64 is."""
    q64, k64, v64 = q.double(), k.double(), v.double()
    share, group, d, n = q.shape[0] // k.shape[0], q.shape[2] // k.shape[2], q.shape[3], k.shape[1]
    k64, v64 = (t.repeat_interleave(share, 0).repeat_interleave(group, 2) for t in (k64, v64))
    s = torch.einsum("sqhd,skhd->shqk", q64, k64) * d ** -0.5
    E = ((d + 8) * U * torch.einsum("sqhd,skhd->shqk", q64.abs(), k64.abs()).amax(-1) * d ** -0.5 + 8 * U)
    want_lse = torch.logsumexp(s, -1)
    p = torch.softmax(s, -1)
    want, mag = torch.einsum("shqk,skhd->sqhd", p, v64), torch.einsum("shqk,skhd->sqhd", p, v64.abs())
    assert torch.equal(torch.isnan(lse), torch.isnan(want_lse)) and torch.equal(torch.isnan(out), torch.isnan(want))
    fine = ~torch.isnan(want_lse)
    assert ((lse.double() - want_lse).abs() <= E + (n + 16) * U + 4 * U * want_lse.abs())[fine].all()
    b, half = (2.0 ** -8 if q.dtype == BF else 0.0), torch.finfo(q.dtype).eps / 2
    bound = mag * (2 * E.transpose(1, 2)[..., None] + (n + 16) * U + b) + half * want.abs() * 1.001
    fine = ~torch.isnan(want)
    assert ((out.double() - want).abs() <= bound)[fine].all()


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_a_query(shape):
    import paper_2511_20390_b200 as free
    q, k, v, g = _inputs(shape)
    q[0, 0, 0] = float("nan")
    q[-1, -1, -1, 3] = float("nan")
    out, lse = free.op_cross_attention(q, k, v, want_lse=True)
    _agrees(out, lse, q, k, v)
    dq, dk, dv = free.op_cross_attention_bwd(q, k, v, out, lse, g)
    hit = torch.isnan(lse).transpose(1, 2)                         # [n_seq, n_q, heads]
    assert hit.sum() == 2
    assert torch.isnan(dq[hit]).all() and torch.isfinite(dq[~hit]).all()
    # the states that such a query reads: all of its key head's
    group, share = q.shape[2] // k.shape[2], q.shape[0] // k.shape[0]
    reach = hit.any(1).view(k.shape[0], share, k.shape[2], group).any(3).any(1)      # [n_enc, kv_heads]
    for t in (dk, dv):
        bad = torch.isnan(t).all(3).all(1)
        assert torch.equal(bad, reach) and torch.isfinite(t.transpose(1, 2)[~reach]).all()


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("where", ["one", "first half", "last 64", "all"])
def test_states(shape, where):
    """Keys with a NaN, among them all those of a part of a split sequence."""
    import paper_2511_20390_b200 as free
    q, k, v, g = _inputs(shape, 2)
    n = k.shape[1]
    at = {"one": slice(n // 3, n // 3 + 1), "first half": slice(0, n // 2), "last 64": slice(n - 64, n), "all": slice(0, n)}[where]
    k[0, at, 0] = float("nan")
    out, lse = free.op_cross_attention(q, k, v, want_lse=True)
    _agrees(out, lse, q, k, v)
    dq, dk, dv = free.op_cross_attention_bwd(q, k, v, out, lse, g)
    hit = torch.isnan(lse).transpose(1, 2)
    assert hit.any() and torch.isnan(dq[hit]).all() and torch.isfinite(dq[~hit]).all()
    assert torch.isnan(dv[0, :, 0]).all() and torch.isnan(dk[0, :, 0]).all()
    keep = torch.ones(k.shape[0], k.shape[2], dtype=torch.bool, device="cuda")
    keep[0, 0] = False
    assert torch.isfinite(dv.transpose(1, 2)[keep]).all() and torch.isfinite(dk.transpose(1, 2)[keep]).all()


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_values_and_what_does_not_count(shape):
    """A value with a NaN: out is NaN in that channel, lse is not.  One in a masked state, or a query without any state: nothing."""
    import paper_2511_20390_b200 as free
    q, k, v, g = _inputs(shape, 3)
    v[0, 5, 0, 1] = float("nan")
    out, lse = free.op_cross_attention(q, k, v, want_lse=True)
    _agrees(out, lse, q, k, v)
    assert torch.isfinite(lse).all() and torch.isnan(out[0, :, 0, 1]).all()
    mask = torch.ones(k.shape[:2], dtype=torch.bool, device="cuda")
    mask[0, 5] = False
    mask[-1] = False if k.shape[0] > 1 else mask[-1]
    if k.shape[0] > 1:
        q[-1] = float("nan")                                       # reads nothing
    out, lse = free.op_cross_attention(q, k, v, kv_mask=mask, want_lse=True)
    assert torch.isfinite(out).all() and not torch.isnan(lse).any()
    dq, dk, dv = free.op_cross_attention_bwd(q, k, v, out, lse, g, kv_mask=mask)
    for t in (dq, dk, dv):
        assert torch.isfinite(t).all()
    assert (dk[0, 5] == 0).all() and (dv[0, 5] == 0).all()
    if k.shape[0] > 1:
        assert (out[-1] == 0).all() and torch.isneginf(lse[-1]).all() and (dq[-1] == 0).all() and (dk[-1] == 0).all() and (dv[-1] == 0).all()
