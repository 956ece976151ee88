"""Packed states of the attention to an encoder's states, against the fp64 definitions with the tolerances of the tests of its shapes:
offsets that leave the rows, sequences of every length, with and without the longest one's."""
import pytest
import torch

import synth
from test_gpu_cross_attention import Case

pytestmark = pytest.mark.gpu


def _case(seed, dt, *shape, lens, **kw):
    """A packed case whose states begin with the first sequence's and end with the last's."""
    c = Case(seed, dt, *shape, lens=lens, layout="packed", **kw)
    c.k, c.v = c.k[3:-5], c.v[3:-5]
    if "kv_mask" in c.kw:
        c.kw["kv_mask"] = c.kw["kv_mask"][3:-5].clone()
    c.kw["kv_offsets"] = c.kw["kv_offsets"] - 3
    c.span = [(slice(s[0].start - 3, s[0].stop - 3),) for s in c.span]
    return c


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("n_q", [1, 70])
def test_offsets_that_leave_the_rows(n_q, dt):
    """A first offset below zero and last ones behind the rows: what is there counts, gradients too."""
    for lens, change in (([50, 0, 100], {0: -7, 3: 1000}), ([60, 90, 0, 0], {0: -1 << 31, 2: 151, 3: 151, 4: (1 << 31) - 1}), ([0, 0, 140], {0: -9, 1: -3, 2: -3})):
        c = _case(3, dt, len(lens), len(lens), n_q, 150, 4, 2, 64, lens=lens)
        for i, v in change.items():
            c.kw["kv_offsets"][i] = v
        c.check()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n_q", [1, 70, 1100])
@pytest.mark.parametrize("most", [0, 20, 64, 130, 300])
def test_rows_behind_the_longest(most, n_q, dt):
    """dk and dv that hold rubbish: rows of a sequence behind the states that may count become zeros, rows of none stay as they are."""
    import paper_2511_20390_b200 as free
    from paper_2511_20390_b200 import binding
    t = lambda role, *s: torch.from_numpy(synth.normal(9, role, s)).to(dt).cuda()
    lens, heads, d = [50, 200, 0, 300], 2, 64
    at = torch.tensor([5, 55, 255, 255, 555], dtype=torch.int32, device="cuda")
    q, g, k, v = t(1, 4, n_q, heads, d), t(2, 4, n_q, heads, d), t(3, 600, heads, d), t(4, 600, heads, d)
    out, lse = free.op_cross_attention(q, k, v, kv_offsets=at, max_kv=most, want_lse=True)
    want = free.op_cross_attention_bwd(q, k, v, out, lse, g, kv_offsets=at, max_kv=most)
    dev, shape = binding._cross_shape(q, k, v, None, None, None, at, most, None)
    dk, dv = (torch.full_like(k, float("nan")) for _ in range(2))
    L = binding.lib()
    need = L.free_op_cross_attention_bwd_workspace_bytes(shape)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")              # NaN too
    qs, ks = q.stride()[:3], (0, *k.stride()[:2])
    assert L.free_op_cross_attention_bwd(shape, out.data_ptr(), *qs, lse.data_ptr(), g.data_ptr(), *qs, None, 0, 0, 0, dk.data_ptr(), *ks, dv.data_ptr(), *ks,
                                         ws.data_ptr(), need, binding._error_word(dev).data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
    assert free.op_device_error() == 0
    for got, ref in ((dk, want[1]), (dv, want[2])):
        assert torch.equal(got[5:555], ref[5:555])
        assert torch.isnan(got[:5]).all() and torch.isnan(got[555:]).all()
        for first, n in zip((5, 55, 255, 255), lens):
            assert (got[first + min(most, n):first + n] == 0).all() and (n_q == 0 or (got[first:first + min(most, n)] != 0).any(2).all())
