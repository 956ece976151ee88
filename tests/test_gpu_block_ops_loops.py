"""The block operators where their kernels go round: more rows than the GPU holds warps, tiles than clusters, tokens than
threads, sequences than CTAs; and every width that chooses another kernel.  Against the fp64 definitions, with the tolerances
derived in the files of the single operators."""
import numpy as np
import pytest
import torch

import synth
import test_gpu_gated_linear as gated
import test_gpu_layer_norm as norm
import test_gpu_rope as rope

pytestmark = pytest.mark.gpu

PAIRS = [("fp32", "bf16"), ("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp32")]

# The norm's forward kernel gives a warp (or a CTA, for wide rows) one row while the GPU holds as many, 4736 warps for the narrowest
# to 148 CTAs for the widest; here each has two rows at least, with groups that begin and end inside its run.
ROUNDS = [  # groups, rows per group, D, extra elements between rows of x
    # four columns per access, widths that whole blocks of 128 columns fill
    (1571, 7, 256, 0), (1900, 5, 384, 0), (740, 11, 512, 0), (1400, 5, 640, 0), (500, 11, 768, 0), (1100, 5, 1024, 0), (620, 7, 1152, 0),
    (400, 11, 1280, 0), (860, 5, 1536, 0), (400, 7, 2048, 0), (560, 5, 2304, 0), (200, 7, 4096, 0), (280, 5, 4608, 0), (65, 11, 8192, 0),
    # the same access, other widths; the last of several warps holds four columns (5124) or nearly all (8188)
    (1700, 5, 392, 0), (640, 11, 600, 0), (800, 7, 900, 4), (1100, 5, 1100, 0), (400, 7, 1300, 0), (280, 5, 4100, 0), (100, 11, 5124, 0),
    (140, 5, 8188, 0),
    # two columns
    (1400, 5, 402, 0), (500, 11, 690, 0), (300, 7, 870, 0), (210, 5, 2050, 0), (700, 5, 1152, 2),
    # one column
    (620, 7, 333, 0), (300, 7, 1001, 0), (210, 5, 2333, 0), (32, 11, 8191, 0),
    # several rows to a warp, or a narrow one
    (2900, 7, 30, 0), (6500, 7, 64, 0), (4400, 5, 100, 0), (1571, 7, 127, 0), (1571, 7, 200, 0), (1571, 7, 255, 0),
]


@pytest.mark.parametrize("xd,yd", PAIRS)
@pytest.mark.parametrize("g,rows,D,pad", ROUNDS)
def test_norm_rows_beyond_the_warps(g, rows, D, pad, xd, yd):
    norm.test_forward_and_backward(g, rows, D, pad, xd, yd)


# The backward kernel's runs of rows inside a group, joined by the second launch, at each of its widths: 12, 16 or 8 columns per lane
# by four, two and one.
RUNS = [
    (3, 1447, 1152, 0), (2, 2001, 640, 0), (2, 1500, 1024, 0), (1, 900, 4100, 0), (1, 701, 8188, 0), (2, 1101, 690, 0), (1, 1203, 870, 0), (1, 800, 4602, 0),
    (1, 3001, 333, 0), (1, 1501, 1001, 0), (2, 900, 512, 1), (1, 1300, 1152, 1), (1, 600, 2048, 1), (1, 700, 4607, 0), (1, 650, 4600, 1), (1, 500, 5001, 0), (1, 400, 8191, 0),
]


@pytest.mark.parametrize("xd,yd", PAIRS)
@pytest.mark.parametrize("g,rows,D,pad", RUNS)
def test_norm_gradients_of_long_groups(g, rows, D, pad, xd, yd):
    norm.test_forward_and_backward(g, rows, D, pad, xd, yd)


# 74 clusters of two CTAs take the tiles of a product: 256 rows x 128 columns of each half forward, 256 x 256 (or 256 x 128) for
# the gradients.  At least three tiles per cluster, whose contraction is longer than the ring of operand stages.
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("M,F,K", [(2000, 2568, 520), (3333, 2056, 72), (130, 28680, 264)])
def test_gated_forward_tiles_beyond_the_clusters(M, F, K, act):
    import paper_2511_20390_b200 as free
    gated._check_forward(free, M, F, K, "bf16", act, bias=F % 16 != 0, seed=M)


@pytest.mark.parametrize("M,F,K,act", [(6100, 328, 2200, "silu"), (600, 2824, 2200, "gelu"), (4173, 1496, 392, "silu"), (20011, 72, 776, "gelu")])
def test_gated_gradient_tiles_beyond_the_clusters(M, F, K, act):
    import paper_2511_20390_b200 as free
    gated._check_backward(free, M, F, K, "bf16", act, seed=M)


@pytest.mark.parametrize("M,F,K,act", [(3001, 700, 130, "silu"), (2500, 513, 64, "gelu")])
def test_gated_fp32_beyond_one_wave(M, F, K, act):
    import paper_2511_20390_b200 as free
    gated._check_forward(free, M, F, K, "fp32", act, seed=M)
    gated._check_backward(free, M, F, K, "fp32", act, seed=M)


# Tokens that a thread unrolls, and sequences that follow one another in a CTA and share its table.
@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("pairing", ["interleaved", "halves"])
@pytest.mark.parametrize("n,t,h,d,axes", [
    (64, 256, 4, 64, (32, 32)), (50, 301, 3, 72, (24, 24, 24)), (3, 4099, 2, 34, (20, 12)), (200, 37, 6, 20, (8, 8)), (33, 129, 40, 128, (48, 40, 40)),
    (90, 64, 2, 256, (128, 128)), (2, 20000, 1, 16, (16,)), (40, 333, 5, 6, (2, 2)),
])
def test_rotary_tokens_and_sequences_of_a_cta(n, t, h, d, axes, pairing, dt):
    import paper_2511_20390_b200 as free
    x = rope._x(n + t, (n, t, h, d), dt)
    pos = torch.from_numpy(np.stack([np.arange(t) // (3 + a) - 5.0 * a for a in range(len(axes))], 1).astype(np.float32)).cuda()
    rope._check(free.op_rope_axes(x, pos, axes, pairing=pairing), x, pos, axes, dt, pairing=pairing)
    each = pos[None] + torch.arange(n, device="cuda")[:, None, None] * 0.5         # positions of every sequence
    got = free.op_rope_axes(x, each, axes, pairing=pairing, joint_freq=True, inverse=True)
    rope._check(got, x, each, axes, dt, pairing=pairing, joint_freq=True, inverse=True)
    # views into a wider matrix whose heads begin at any element, and in place
    wide = torch.zeros(n, t, h + 1, d + 2, dtype=x.dtype, device="cuda")
    wide[:, :, :h, :d] = x
    view = wide[:, :, :h, :d]
    free.op_rope_axes(view, pos, axes, pairing=pairing, out=view)
    rope._check(view, x, pos, axes, dt, pairing=pairing)
    assert not wide[:, :, h].any() and not wide[..., d:].any()


def test_rotary_more_sequences_than_a_grid_dimension():
    # 70001 sequences, each with positions of its own: a CTA fills its table again for its second one
    import paper_2511_20390_b200 as free
    n = 70001
    x = rope._x(9, (n, 2, 1, 8), "fp32")
    pos = torch.from_numpy(synth.normal(9, 2, (n, 2, 2)) * np.float32(50)).cuda()
    for pairing in ("interleaved", "halves"):
        rope._check(free.op_rope_axes(x, pos, (4, 4), pairing=pairing), x, pos, (4, 4), "fp32", pairing=pairing)
