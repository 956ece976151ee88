"""Packed states of the attention to an encoder's states, against the fp64 definitions with the tolerances of the tests of its shapes:
offsets that leave the rows, sequences of every length, with and without the longest one's."""
import pytest
import torch

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
