"""The attention to an encoder's states and the RMS norm as a text-conditioned block uses them together, forward and backward, against
the fp64 definitions; and what calls meet outside a quiet stream: captures, other streams, layouts, lengths of zero, long caches."""
import numpy as np
import pytest
import torch
import torch.nn.functional as TF

import synth
from gpu_util import rms_rel

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _t(seed, role, shape, dt, scale=1.0):
    return torch.from_numpy((synth.normal(seed, role, shape) * np.float32(scale)).astype(np.float32)).to(dt).cuda()


def _rms64(x, w, eps=1e-6):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * w


def _cross64(q, k, v, lens, share):
    """[n_seq, n_q, heads, d] over [n_enc, n_kv, heads, d] in fp64."""
    group = q.shape[2] // k.shape[2]
    k, v = (t.repeat_interleave(share, 0).repeat_interleave(group, 2) for t in (k, v))
    s = torch.einsum("sqhd,skhd->shqk", q, k) * q.shape[-1] ** -0.5
    dead = torch.arange(k.shape[1], device=q.device)[None, :] >= torch.tensor(lens, device=q.device).repeat_interleave(share)[:, None]
    p = torch.softmax(s.masked_fill(dead[:, None, None], -torch.inf), -1)
    return torch.einsum("shqk,skhd->sqhd", torch.nan_to_num(p, nan=0.0), v)


@pytest.mark.parametrize("dt,tol", [(torch.bfloat16, 2e-2), (torch.float32, 2e-5)])
@pytest.mark.parametrize("n_seq,n_enc,T,S,heads,kvh,dh,lens", [(6, 2, 256, 120, 6, 6, 64, [120, 37]), (2, 2, 100, 77, 8, 2, 72, [0, 77]), (3, 3, 1, 300, 4, 4, 48, [300, 1, 200])])
def test_conditioned_block(n_seq, n_enc, T, S, heads, kvh, dh, lens, dt, tol):
    # 2e-2: the framework's bound for bf16 passes; fp32: sums of at most a thousand terms, a handful of them in a row
    import paper_2511_20390_b200 as free
    from paper_2511_20390_b200 import binding
    D, M, code = heads * dh, n_seq * T, binding._code(dt)
    x, a = _t(1, 1, (M, D), torch.float32), _t(1, 2, (M, D), dt)
    text = _t(1, 3, (n_enc * S, D), dt)
    w1, wq_n, wk_n, w2 = (1 + _t(1, 4 + i, (n,), torch.float32, 0.2) for i, n in enumerate((D, dh, dh, D)))
    wq, wkv, wo = _t(1, 8, (D, D), dt, D ** -0.5), _t(1, 9, (2 * kvh * dh, D), dt, D ** -0.5), _t(1, 10, (D, D), dt, D ** -0.5)
    lens_t = torch.tensor(lens, dtype=torch.int32, device="cuda")
    # the attention's result joins the stream, norm; queries and keys normed by heads, the keys in place inside the packed projection
    n1 = free.op_rms_norm(a, w1, residual=x, out_dtype=dt, want_rstd=True)
    q = free.op_linear(n1.y, wq, out_dtype=code).view(M, heads, dh)
    qn = free.op_rms_norm(q, wq_n, want_rstd=True)
    kv = free.op_linear(text, wkv, out_dtype=code).view(n_enc * S, 2 * kvh, dh)
    k_raw = kv[:, :kvh].clone()
    kn = free.op_rms_norm(kv[:, :kvh], wk_n, want_rstd=True, out=kv[:, :kvh])
    kv4 = kv.view(n_enc, S, 2, kvh, dh)
    k, v, q4 = kv4[:, :, 0], kv4[:, :, 1], qn.y.view(n_seq, T, heads, dh)
    out, lse = free.op_cross_attention(q4, k, v, kv_lens=lens_t, want_lse=True)
    o = free.op_linear(out.view(M, D), wo, out_dtype=code)
    n2 = free.op_rms_norm(o, w2, residual=n1.residual, residual_out=n1.residual, out_dtype=dt)
    assert n2.residual is n1.residual
    n8 = free.op_rms_norm(o, w2, out_dtype=torch.float8_e4m3fn, scale_block=128)
    # backward, from a gradient of the attention's result
    g = _t(1, 11, (n_seq, T, heads, dh), dt, 0.1)
    dq, dk, dv = free.op_cross_attention_bwd(q4, k, v, out, lse, g, kv_lens=lens_t)
    dqr, dwq = free.op_rms_norm_bwd(q, dq.view(M, heads, dh), qn.rstd, wq_n)
    dkr, dwk = free.op_rms_norm_bwd(k_raw, dk.view(n_enc * S, kvh, dh), kn.rstd, wk_n)
    assert free.op_device_error() == 0

    f = lambda t: t.double()
    h = f(x) + f(a)
    y = _rms64(h, f(w1))
    q64, kv64 = (y @ f(wq).T).view(M, heads, dh), (f(text) @ f(wkv).T).view(n_enc, S, 2, kvh, dh)
    leaves = [t.detach().requires_grad_() for t in (q64, kv64[:, :, 0], kv64[:, :, 1], f(wq_n), f(wk_n))]
    o64 = _cross64(_rms64(leaves[0], leaves[3]).view(n_seq, T, heads, dh), _rms64(leaves[1], leaves[4]), leaves[2], lens, n_seq // n_enc)
    grads = torch.autograd.grad(o64, leaves, f(g))
    res = h + o64.detach().reshape(M, D) @ f(wo).T
    y2 = _rms64(res, f(w2))
    c = lambda t: t.double().cpu().numpy()
    for got, want in ((out, o64), (n2.residual, res), (n2.y, y2), (dqr, grads[0]), (dkr, grads[1]), (dv, grads[2]), (dwq, grads[3]), (dwk, grads[4])):
        assert rms_rel(c(got).reshape(-1), c(want.detach()).reshape(-1)) < tol, (rms_rel(c(got).reshape(-1), c(want.detach()).reshape(-1)))
    # 8-bit values times their scales: a rounding of 2^-4 of the value, or half a step of 2^-9 of the scale, beside the rest
    y8 = _rms64(f(o), f(w2))
    back = f(n8.y) * f(n8.scales).repeat_interleave(128, 1)[:, :D]
    assert ((back - y8).abs() <= (2.0 ** -4 + 1e-5) * y8.abs() + 2.0 ** -10 * f(n8.scales).repeat_interleave(128, 1)[:, :D] * 1.01).all()


def test_gradients_are_those_of_differences():
    """Central differences of the fp32 calls along random directions.  The difference quotient is off by the rounding of both results
    over the step, and by its third derivative, which the quotient of twice the step shows four times over."""
    import paper_2511_20390_b200 as free
    q, k, v = (_t(3, i, s, torch.float32) for i, s in enumerate(((2, 9, 4, 24), (2, 21, 2, 24), (2, 21, 2, 24))))
    lens = torch.tensor([21, 13], dtype=torch.int32, device="cuda")
    r = _t(3, 5, q.shape, torch.float32)
    out, lse = free.op_cross_attention(q, k, v, kv_lens=lens, want_lse=True)
    grads = free.op_cross_attention_bwd(q, k, v, out, lse, r, kv_lens=lens)
    f = lambda *a: (free.op_cross_attention(*a, kv_lens=lens).double() * r.double()).sum().item()
    _differences(f, [q, k, v], grads, 100 * U * (r.abs().sum() * v.abs().max()).item())
    x, w = _t(3, 6, (37, 72), torch.float32), 1 + _t(3, 7, (72,), torch.float32, 0.3)
    r2 = _t(3, 8, x.shape, torch.float32)
    y = free.op_rms_norm(x, w, want_rstd=True)
    grads = free.op_rms_norm_bwd(x, r2, y.rstd, w)
    f = lambda a, b: (free.op_rms_norm(a, b).y.double() * r2.double()).sum().item()
    _differences(f, [x, w], [grads[0], grads[1][0]], 40 * U * (y.y.abs() * r2.abs()).sum().item())


def _differences(f, args, grads, rounding):
    step = 2.0 ** -8
    for i, g in enumerate(grads):
        u = _t(4, i, tuple(args[i].shape), torch.float32)
        quotient = lambda e: (f(*[a + e * u if j == i else a for j, a in enumerate(args)]) - f(*[a - e * u if j == i else a for j, a in enumerate(args)])) / (2 * e)
        d1, d2 = quotient(step), quotient(2 * step)
        want = (g.double() * u.double()).sum().item()
        # (arguments a + e u are rounded too: U of them, times their gradients)
        bound = rounding / step + abs(d2 - d1) + 4 * U / step * (g.abs() * args[i].abs()).sum().item() + 1e-5 * (g.abs() * u.abs()).sum().item()
        assert abs(want - d1) <= bound, (i, want, d1, bound)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", [(4, 2, 130, 90, 4, 2, 64), (2, 2, 1, 5000, 4, 4, 128), (3, 1, 200, 150, 2, 2, 72)], ids=str)
def test_streams_and_graphs(shape, dt):
    import paper_2511_20390_b200 as free
    n_seq, n_enc, n_q, n_kv, heads, kvh, d = shape
    q, g = _t(5, 1, (n_seq, n_q, heads, d), dt), _t(5, 2, (n_seq, n_q, heads, d), dt, 0.1)
    k, v = _t(5, 3, (n_enc, n_kv, kvh, d), dt), _t(5, 4, (n_enc, n_kv, kvh, d), dt)
    lens = torch.tensor([n_kv, 0][:n_enc], dtype=torch.int32, device="cuda")
    w = 1 + _t(5, 6, (d,), torch.float32, 0.1)

    def run():
        qn = free.op_rms_norm(q.view(-1, heads, d), w, want_rstd=True)
        qn4 = qn.y.view(q.shape)
        out, lse = free.op_cross_attention(qn4, k, v, kv_lens=lens, want_lse=True)
        dq, dk, dv = free.op_cross_attention_bwd(qn4, k, v, out, lse, g, kv_lens=lens)
        return (out, lse, dk, dv) + free.op_rms_norm_bwd(q.view(-1, heads, d), dq.view(-1, heads, d), qn.rstd, w)

    same = lambda a, b: all(torch.equal(x, y) for x, y in zip(a, b))
    ref = run()
    torch.cuda.synchronize()
    outs = []
    for s in [torch.cuda.Stream() for _ in range(3)]:              # several at once: every call has its own workspace
        with torch.cuda.stream(s):
            outs.append(run())
    torch.cuda.synchronize()
    assert all(same(o, ref) for o in outs)
    graphs = []
    for _ in range(2):                                             # two captured graphs, replayed one behind the other
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = run()
        graphs.append((graph, got))
    q.mul_(0.5); g.neg_(); lens.copy_(torch.tensor([n_kv // 2, n_kv][:n_enc], dtype=torch.int32)); k[:, :3].add_(1)
    for _ in range(2):
        for graph, _ in graphs:
            graph.replay()
    torch.cuda.synchronize()
    want = run()
    assert not same(want, ref) and all(same(got, want) for _, got in graphs)
    assert free.op_device_error() == 0


def test_first_call_inside_a_capture_is_refused():
    from paper_2511_20390_b200 import binding
    q, k = torch.zeros(1, 4, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 4, 2, 64, dtype=torch.bfloat16, device="cuda")
    kept = dict(binding._ERROR_WORDS)
    binding._ERROR_WORDS.clear()
    refused = False
    try:
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            try:
                binding.op_cross_attention(q, k, k)
            except RuntimeError:
                refused = True
            q.add_(0.0)                                            # a graph with something in it
    finally:
        binding._ERROR_WORDS.update(kept)
    assert refused
    assert not binding.op_cross_attention(q, k, k).any()


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n_q,n_kv,d", [(1, 300, 64), (150, 200, 72), (70, 65, 128)])
def test_layouts(n_q, n_kv, d, dt):
    """Heads before tokens in memory, states and heads that several share by strides of zero, a result inside another tensor."""
    import paper_2511_20390_b200 as free
    n_seq, heads = 4, 4
    q = _t(6, 1, (n_seq, heads, n_q, d), dt).transpose(1, 2)
    g = _t(6, 2, (heads, n_seq, n_q, d), dt, 0.1).permute(1, 2, 0, 3)
    kv = _t(6, 3, (2, n_kv, 2, d), dt)
    same = lambda a, b: all(torch.equal(x, y) for x, y in zip(a, b))
    for k, v in ((kv[0][None].expand(n_seq, -1, -1, -1), kv[1][None].expand(n_seq, -1, -1, -1)),
                 (kv[0, None, :, :1].expand(n_seq, -1, heads, -1), kv[1, None, :, 1:].expand(n_seq, -1, heads, -1)),
                 (kv[0].transpose(0, 1).contiguous().transpose(0, 1)[None].expand(n_seq, -1, -1, -1), kv[1][None].expand(n_seq, -1, -1, -1))):
        qc, kc, vc, gc = (t.contiguous() for t in (q, k, v, g))
        out, lse = free.op_cross_attention(qc, kc, vc, want_lse=True)
        into = torch.full((n_seq, n_q, 3, heads, d), 7.0, dtype=dt, device="cuda")
        out2, lse2 = free.op_cross_attention(q, k, v, want_lse=True, out=into[:, :, 1])
        assert torch.equal(out, out2) and torch.equal(lse, lse2) and (into[:, :, 0] == 7).all() and (into[:, :, 2] == 7).all()
        assert same(free.op_cross_attention_bwd(q, k, v, out2, lse, g), free.op_cross_attention_bwd(qc, kc, vc, out, lse, gc))
    # one byte per state, whatever type it has
    mask = torch.from_numpy(synth.normal(6, 9, (n_seq, n_kv)) > 0).cuda()
    assert torch.equal(free.op_cross_attention(q, k, v, kv_mask=mask), free.op_cross_attention(q, k, v, kv_mask=mask.to(torch.uint8) * 3))


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n_q", [1, 7, 140])
def test_results_one_by_one_and_elsewhere(n_q, dt):
    """Either gradient without the other, no lse, heads before tokens in the result: the same numbers."""
    import paper_2511_20390_b200 as free
    q, g = _t(10, 1, (4, n_q, 6, 64), dt), _t(10, 2, (4, n_q, 6, 64), dt)
    k, v = _t(10, 3, (2, 200, 3, 64), dt), _t(10, 4, (2, 200, 3, 64), dt)
    out, lse = free.op_cross_attention(q, k, v, want_lse=True)
    assert torch.equal(free.op_cross_attention(q, k, v), out)
    assert torch.equal(free.op_cross_attention(q, k, v, out=torch.empty(4, 6, n_q, 64, dtype=dt, device="cuda").transpose(1, 2)), out)
    assert torch.equal(free.op_cross_attention(q, k, v, out=torch.empty(n_q, 6, 4, 64, dtype=dt, device="cuda").permute(2, 0, 1, 3)), out)
    dq, dk, dv = free.op_cross_attention_bwd(q, k, v, out, lse, g)
    one = free.op_cross_attention_bwd(q, k, v, out, lse, g, want_dkv=False)
    two = free.op_cross_attention_bwd(q, k, v, out, lse, g, want_dq=False)
    assert one[1] is None and one[2] is None and two[0] is None
    assert torch.equal(one[0], dq) and torch.equal(two[1], dk) and torch.equal(two[2], dv)
    assert free.op_cross_attention_bwd(q, k, v, out, lse, g, want_dq=False, want_dkv=False) == (None, None, None)
    # one sequence of states for all, read in an order of its own, is what every sequence's own copy gives
    seq = torch.tensor([1, 0, 0, 1], dtype=torch.int32, device="cuda")
    got, lse2 = free.op_cross_attention(q, k, v, kv_seq=seq, want_lse=True)
    pick = seq.long()
    assert torch.equal(got, free.op_cross_attention(q, k[pick], v[pick]))
    dks = free.op_cross_attention_bwd(q, k[pick], v[pick], got, lse2, g)[1].double()
    dk2 = free.op_cross_attention_bwd(q, k, v, got, lse2, g, kv_seq=seq)[1].double()
    # every copy's gradient is rounded, and their sum: half a step each; and sums of 4 n_q terms at most run in another order
    f = lambda t: t.double().repeat_interleave(2, 2) if t.shape[2] == 3 else t.double()
    p = torch.softmax(torch.einsum("sqhd,skhd->shqk", f(q), f(k[pick])) / 8, -1)
    ds = p * (torch.einsum("sqhd,skhd->shqk", f(g), f(v[pick])) - (f(g) * f(got)).sum(-1).transpose(1, 2)[..., None]) / 8
    terms = torch.einsum("shqk,sqhd->skhd", ds.abs(), f(q).abs()).view(4, 200, 3, 2, 64).sum(3)
    half = torch.finfo(dt).eps / 2
    add = lambda t: torch.zeros_like(dk2).index_add(0, pick, t)
    want = add(dks)
    assert ((dk2 - want).abs() <= half * 1.01 * (add(dks.abs()) + want.abs()) + (8 * n_q + 32) * U * add(terms) + 1e-30).all()


@pytest.mark.parametrize("n_q,d", [(1, 36), (100, 36), (150, 20), (90, 68), (70, 100), (130, 127)])
def test_heads_with_gaps(n_q, d):
    """Head sizes of no whole 16 bytes whose heads lie 16-byte aligned take the tensor cores; dense ones do not.  Both round p and dS or
    the results to bf16 (2^-8 of each term, which add up like errors of either sign): 1e-2 in the 2-norm."""
    import paper_2511_20390_b200 as free
    n_seq, n_kv, heads, kvh = 2, 150, 4, 2
    wide = lambda role, *s: _t(9, role, (*s, (d + 7) // 8 * 8), torch.bfloat16)[..., :d]
    q, g, k, v = wide(1, n_seq, n_q, heads), wide(2, n_seq, n_q, heads), wide(3, n_seq, n_kv, kvh), wide(4, n_seq, n_kv, kvh)
    lens = torch.tensor([150, 70], dtype=torch.int32, device="cuda")
    out = torch.full((n_seq, n_q, heads, (d + 7) // 8 * 8), 7.0, dtype=torch.bfloat16, device="cuda")
    got, lse = free.op_cross_attention(q, k, v, kv_lens=lens, want_lse=True, out=out[..., :d])
    c = lambda t: t.double().cpu().numpy()
    f = lambda t: t.double().requires_grad_()
    leaves = [f(q), f(k), f(v)]
    want = _cross64(*leaves, [150, 70], 1)
    assert rms_rel(c(got), c(want.detach())) < 1e-2 and (out[..., d:] == 7).all()
    for a, b in zip(free.op_cross_attention_bwd(q, k, v, got, lse, g, kv_lens=lens), torch.autograd.grad(want, leaves, g.double())):
        assert rms_rel(c(a), c(b)) < 1e-2
    assert free.op_device_error() == 0


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n_q", [1, 70])
def test_lengths_that_say_too_much(n_q, dt):
    """Lengths below zero or above the room, offsets that run backwards or out of the states: what is there counts."""
    import paper_2511_20390_b200 as free
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    q, g = _t(7, 1, (3, n_q, 2, 64), dt), _t(7, 2, (3, n_q, 2, 64), dt)
    k, v = _t(7, 3, (3, 50, 2, 64), dt), _t(7, 4, (3, 50, 2, 64), dt)
    kp, vp = k.view(150, 2, 64), v.view(150, 2, 64)

    def both(k, v, **kw):
        out, lse = free.op_cross_attention(q, k, v, want_lse=True, **kw)
        return (out, lse) + free.op_cross_attention_bwd(q, k, v, out, lse, g, **kw)
    same = lambda a, b: all(torch.equal(x, y) for x, y in zip(a, b))
    assert same(both(k, v, kv_lens=i32(-5, 1 << 30, 20)), both(k, v, kv_lens=i32(0, 50, 20)))
    got = both(kp, vp, kv_offsets=i32(-7, 50, 40, 1000))
    one = lambda s, a, b: free.op_cross_attention(q[s:s + 1], kp[a:b], vp[a:b], kv_offsets=i32(0, b - a), want_lse=True)
    for s, (a, b) in enumerate(((0, 50), (40, 40), (40, 150))):
        if a == b:
            assert (got[0][s] == 0).all() and torch.isneginf(got[1][s]).all()
            continue
        want = one(s, a, b)
        assert torch.allclose(got[0][s:s + 1].float(), want[0].float(), atol=2e-2 if dt == torch.bfloat16 else 1e-5)
    # max_kv cuts every sequence
    cut = both(kp, vp, kv_offsets=i32(0, 50, 100, 150), max_kv=20)
    assert torch.equal(cut[0], both(k, v, kv_lens=i32(20, 20, 20))[0])
    assert (cut[3].view(3, 50, 2, 64)[:, 20:] == 0).all()


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_nothing(dt):
    import paper_2511_20390_b200 as free
    mk = lambda *s: torch.randn(*s, device="cuda").to(dt)
    for q, k in ((mk(0, 5, 2, 64), mk(0, 7, 2, 64)), (mk(0, 5, 2, 64), mk(3, 7, 2, 64)), (mk(3, 0, 2, 64), mk(3, 7, 2, 64)), (mk(3, 5, 2, 64), mk(3, 0, 2, 64))):
        out, lse = free.op_cross_attention(q, k, k, want_lse=True)
        assert out.shape == q.shape and (out == 0).all() and torch.isneginf(lse).all()
        dq, dk, dv = free.op_cross_attention_bwd(q, k, k, out, lse, q)
        assert (dq == 0).all() and (dk == 0).all() and (dv == 0).all() and dk.shape == k.shape
    x = mk(0, 64)
    y = free.op_rms_norm(x, want_rstd=True)
    assert y.y.shape == x.shape and free.op_rms_norm_bwd(x, x, y.rstd)[0].shape == x.shape
    y = free.op_rms_norm(mk(0, 64), torch.ones(64, device="cuda"), out_dtype=torch.float8_e4m3fn)
    assert y.scales.shape == (0, 1)
    dx, dw = free.op_rms_norm_bwd(x, x, torch.empty(0, device="cuda"), torch.ones(64, device="cuda"))
    assert (dw == 0).all()


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_rows_of_no_sequence_are_left_alone(dt):
    """The library's own call on packed states: rows in front of the first sequence and behind the last keep what they held."""
    import paper_2511_20390_b200 as free
    from paper_2511_20390_b200 import binding as b
    q, k, v = _t(8, 1, (2, 40, 2, 64), dt), _t(8, 2, (90, 2, 64), dt), _t(8, 3, (90, 2, 64), dt)
    at = torch.tensor([4, 30, 80], dtype=torch.int32, device="cuda")
    out, lse = free.op_cross_attention(q, k, v, kv_offsets=at, want_lse=True)
    want = free.op_cross_attention_bwd(q, k, v, out, lse, q, kv_offsets=at)
    dev, shape = b._cross_shape(q, k, v, None, None, None, at, None, None)
    dk, dv = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    ws = torch.full((b.lib().free_op_cross_attention_bwd_workspace_bytes(shape),), 255, dtype=torch.uint8, device="cuda")
    qs, ks = q.stride()[:3], (0, *k.stride()[:2])
    b._launch("free_op_cross_attention_bwd", dev, shape, out.data_ptr(), *qs, lse.data_ptr(), q.data_ptr(), *qs, None, 0, 0, 0, dk.data_ptr(), *ks, dv.data_ptr(), *ks,
              ws.data_ptr(), ws.numel(), b._error_word(dev).data_ptr())
    for got, full in ((dk, want[1]), (dv, want[2])):
        assert torch.equal(got[4:80], full[4:80]) and (got[:4] == 7).all() and (got[80:] == 7).all()


@pytest.mark.parametrize("n_q", [1, 40])
def test_states_behind_the_31st_bit(n_q):
    """A cache of more than 2^31 elements: its last states count as the first do."""
    import paper_2511_20390_b200 as free
    n_kv, kvh, d = (1 << 21) + 77, 8, 128
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    kv = torch.zeros(1, n_kv, 2, kvh, d, dtype=torch.bfloat16, device="cuda")
    q = torch.full((1, n_q, kvh, d), 1.0, dtype=torch.bfloat16, device="cuda")
    for j in (0, n_kv - 1):
        kv[0, j, 0] = 8.0                                          # a score of 8 sqrt(128) = 90: the others' weights are e^-90
        kv[0, j, 1] = 2.0 + (j > 0)
    out = free.op_cross_attention(q, kv[:, :, 0], kv[:, :, 1])
    assert (out == 2.5).all()
    lens = torch.tensor([n_kv - 1], dtype=torch.int32, device="cuda")
    assert (free.op_cross_attention(q, kv[:, :, 0], kv[:, :, 1], kv_lens=lens) == 2.0).all()
    assert (free.op_cross_attention(q, kv[0, :, 0], kv[0, :, 1], kv_offsets=torch.tensor([1, n_kv], dtype=torch.int32, device="cuda")) == 3.0).all()
    assert free.op_device_error() == 0


def test_binding_refuses():
    import paper_2511_20390_b200 as free
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    q, k = bf(4, 5, 2, 64), bf(2, 9, 2, 64)
    out, lse = free.op_cross_attention(q, k, k, want_lse=True)
    f = free.op_cross_attention
    for call in (
            lambda: f(q, k, k, kv_lens=torch.tensor([1, 2], device="cuda")), lambda: f(q, k, k, kv_lens=i32(1, 2, 3)), lambda: f(q, k, k, kv_lens=torch.tensor([1, 2], dtype=torch.int32)),
            lambda: f(q, k, k, kv_mask=torch.ones(2, 8, dtype=torch.bool, device="cuda")), lambda: f(q, k, k, kv_mask=torch.ones(9, 2, dtype=torch.bool, device="cuda").T),
            lambda: f(q, k, k, kv_seq=i32(0, 1)), lambda: f(q[:3], k, k), lambda: f(q, k, k, max_kv=3), lambda: f(q, k, k, out=q), lambda: f(q, k, k, out=q.float()),
            lambda: f(q, k[0], k[0], kv_offsets=i32(0, 9), kv_lens=i32(9)), lambda: f(q, k[0], k[0], kv_offsets=i32(0, 9), max_kv=-1),
            lambda: f(q, k[..., ::2], k[..., ::2]), lambda: f(q, k, k.float()), lambda: f(q.half(), k.half(), k.half()),
            lambda: free.op_cross_attention_bwd(q, k, k, out, lse[:, :1], q), lambda: free.op_cross_attention_bwd(q, k, k, out, lse, q[:, :3]),
            lambda: free.op_cross_attention_bwd(q, k, k, out.float(), lse, q)):
        with pytest.raises(ValueError):
            call()
    for kw in ({"scale": 0.0}, {"scale": float("nan")}):
        with pytest.raises(free.FreeError):
            f(q, k, k, **kw)
    with pytest.raises(free.FreeError):
        f(bf(4, 5, 3, 64), k, k)                                   # heads that share no whole number of key heads
    with pytest.raises(free.FreeError):
        f(bf(4, 5, 2, 136), bf(2, 9, 2, 136), bf(2, 9, 2, 136))
    x, w = bf(6, 64), torch.ones(64, device="cuda")
    r = free.op_rms_norm
    for call in (lambda: r(x, w[:32]), lambda: r(x, w.bfloat16()), lambda: r(x, residual=bf(5, 64)), lambda: r(x, residual_out=x), lambda: r(x, scale_block=128),
                 lambda: r(x, out_dtype=torch.float8_e4m3fn, scale_block=64), lambda: r(x.view(6, 2, 32), residual=x), lambda: r(x.view(6, 2, 32), out_dtype=torch.float8_e4m3fn),
                 lambda: r(x, out_dtype=torch.float16), lambda: r(x.half()), lambda: r(x, out=bf(6, 32)), lambda: r(x[:4], out=x[1:5]),
                 lambda: r(x, residual=x.clone(), residual_out=x[:3]), lambda: free.op_rms_norm_bwd(x, x, torch.ones(5, device="cuda")),
                 lambda: free.op_rms_norm_bwd(x, x, torch.ones(6, device="cuda"), dres=x.float())):
        with pytest.raises(ValueError):
            call()
