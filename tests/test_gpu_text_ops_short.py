"""Gradients of the attention to an encoder's states for many sequences of one or a few tokens whose matrices have gaps: the same numbers as
without gaps, in about the same time."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _call(n_seq, n_q, heads, d, dt):
    """Calls with a dense gradient and with the same one inside a larger matrix."""
    import paper_2511_20390_b200 as free
    q, k = torch.randn(n_seq, n_q, heads, d, device="cuda").to(dt), torch.randn(n_seq, 3, heads, d, device="cuda").to(dt)
    g = torch.randn(n_seq, n_q, 2, heads, d, device="cuda").to(dt)
    out, lse = free.op_cross_attention(q, k, k, want_lse=True)
    dense = g[:, :, 0].contiguous()
    return [lambda x=x: free.op_cross_attention_bwd(q, k, k, out, lse, x, want_dkv=False)[0] for x in (dense, g[:, :, 0])], (q, k, dense)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", [(40000, 1, 1, 64), (30000, 2, 1, 20), (9001, 3, 5, 8), (5000, 7, 3, 72), (3, 1, 2, 64), (700, 2, 40, 128)], ids=str)
def test_the_same_gradients(shape, dt):
    (a, b), (q, k, g) = _call(*shape, dt)
    x, y = a(), b()
    assert torch.equal(x, y)
    # and those of the formula, at 32-bit inputs; a sum of d products and one of three states: a few hundred roundings of 2^-24
    if dt == torch.float32:
        q, k, g = q.double().transpose(1, 2), k.double().transpose(1, 2), g.double().transpose(1, 2)
        scale = shape[3] ** -0.5
        p = torch.softmax(q @ k.transpose(2, 3) * scale, -1)
        dp = g @ k.transpose(2, 3)
        ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * scale
        size = p * scale * (g.abs() @ k.abs().transpose(2, 3) + (p * dp.abs()).sum(-1, keepdim=True))
        spread = (q.abs() @ k.abs().transpose(2, 3)).amax(-1, keepdim=True) * scale
        assert ((x.double().transpose(1, 2) - ds @ k).abs() <= 2.0 ** -24 * (2 * (shape[3] + 8) * (1 + spread) + 64) * (size @ k.abs())).all()


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_in_about_the_same_time(dt):
    """One token each (rows were counted on by subtracting its length over and over: 3 to 16 times as long)."""
    calls, _ = _call(32768, 1, 1, 64, dt)
    best = [1e30, 1e30]
    for _ in range(6):
        for i, f in enumerate(calls):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            f()
            f()
            b.record()
            b.synchronize()
            best[i] = min(best[i], a.elapsed_time(b))
    assert best[1] <= 1.5 * best[0]
