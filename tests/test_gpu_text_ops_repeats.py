"""Repeats of the attention to an encoder's states are bit-identical whatever ran before: groups of query heads that leave rows of a tile of 128
unused, after calls that leave other numbers in shared memory."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(10, 10, 105, 300, 12, 4, 72), (6, 6, 190, 520, 5, 1, 128), (40, 8, 60, 400, 6, 1, 40), (4, 4, 130, 700, 14, 2, 64), (3, 3, 90, 900, 3, 1, 120),
                                   (2, 2, 40, 600, 40, 1, 96), (2, 1, 30, 500, 100, 1, 64), (3, 3, 100, 4100, 5, 1, 80)], ids=str)
def test_groups_that_leave_rows_of_a_tile(shape):
    import paper_2511_20390_b200 as free
    n_seq, n_enc, n_q, n_kv, heads, kvh, d = shape
    gen = torch.Generator("cuda").manual_seed(1)
    mk = lambda *s: torch.randn(*s, device="cuda", generator=gen).to(torch.bfloat16)
    # scores that grow along the states, so that rows move their maxima block after block
    q, k, v = mk(n_seq, n_q, heads, d), mk(n_enc, n_kv, kvh, d), mk(n_enc, n_kv, kvh, d)
    k *= torch.linspace(0.2, 6, n_kv, device="cuda")[:, None, None].to(torch.bfloat16)
    want, lse = free.op_cross_attention(q, k, v, want_lse=True)
    for i in range(12):
        # every CTA's tiles full of other numbers
        other = [mk(300, 128, 1, d) * 2.0 ** (i % 5 - 2), mk(300, 300, 1, d) * 4, mk(300, 300, 1, d)]
        free.op_cross_attention(*other)
        out, again = free.op_cross_attention(q, k, v, want_lse=True)
        assert torch.equal(out, want) and torch.equal(again, lse), i
    assert free.op_device_error() == 0
