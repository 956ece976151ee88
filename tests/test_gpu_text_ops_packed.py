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
@pytest.mark.parametrize("most", [0, 20, 64, 130, 250, 260, 300])
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


EDGES = [0, 1, 63, 64, 65, 127, 128, 129, 191, 192, 193, 255, 256, 257]


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("longest", [False, True])
def test_lengths_around_whole_blocks(dt, longest):
    """Blocks of states of every sequence, whatever the sequences before it leave of a block; few sequences and more than a warp finds at once."""
    for lens in (EDGES, EDGES[::-1], [129] * 5, [1] * 70, [0] * 40 + [128] + [0] * 40, [300] + [0] * 33 + [1, 127, 1]):
        c = Case(5, dt, len(lens), len(lens), 9, max(lens), 2, 2, 32, lens=lens, layout="packed", mask=len(lens) == 14)
        if longest:
            c.kw["max_kv"] = max(lens)
        c.check()


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
def test_more_sequences_than_blocks_at_once(dt):
    """1100 short sequences, read in another order, some of them by several tokens' sequences."""
    lens = [(7 * e) % 23 for e in range(1100)]
    Case(6, dt, 40, 1100, 5, 22, 2, 1, 16, lens=lens, layout="packed", seq_of=[(e * 37) % 1100 for e in range(40)]).check()


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("n_q", [20, 1100])
def test_few_sequences_in_many_rows(n_q, dt):
    """Rows of which the offsets name a few, far from the first: the others' gradients are zero.  Many tokens: in parts."""
    c = Case(7, dt, 3, 3, n_q, 150, 2, 2, 64, lens=[150, 0, 77], layout="packed")
    at = 40000
    far = torch.full((100000, 2, 2, 64), float("nan"), dtype=c.k.dtype, device="cuda")
    far[at:at + len(c.k), 0], far[at:at + len(c.k), 1] = c.k, c.v
    c.k, c.v = far[:, 0], far[:, 1]
    c.kw["kv_offsets"] = c.kw["kv_offsets"] + at
    c.span = [(slice(s[0].start + at, s[0].stop + at),) for s in c.span]
    c.check()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_work_grows_with_the_rows(dt):
    """512 sequences of 48 to 64 states: without their longest length the gradients take no more than twice what they take with it (blocks were
    found by walking over as many of every sequence as all rows together make: 5 to 20 times)."""
    import paper_2511_20390_b200 as free
    lens = [64 - e % 17 for e in range(512)]
    at = torch.tensor([0] + lens).cumsum(0).int().cuda()
    q, g = (torch.randn(512, 64, 8, 64, device="cuda").to(dt) for _ in range(2))
    k, v = (torch.randn(sum(lens), 8, 64, device="cuda").to(dt) for _ in range(2))

    def took(m):
        out, lse = free.op_cross_attention(q, k, v, kv_offsets=at, max_kv=m, want_lse=True)
        best = 1e30
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(3):
                free.op_cross_attention_bwd(q, k, v, out, lse, g, kv_offsets=at, max_kv=m)
            b.record()
            b.synchronize()
            best = min(best, a.elapsed_time(b))
        return best
    assert took(None) <= 2 * took(64)
