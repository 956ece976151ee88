"""The root-mean-square norm at every width that chooses another kernel: whole blocks of 128 columns and their neighbours, heads up to 128 columns,
each in the types that choose between accesses of 16 and 8 bytes, with the checks and tolerances of the tests of its shapes."""
import pytest

import test_gpu_rms_norm as base

pytestmark = pytest.mark.gpu
WIDTHS = [n * 128 for n in range(1, 11)] + [136, 248, 264, 376, 504, 520, 632, 648, 888, 1016, 1032, 1144, 1160]


@pytest.mark.parametrize("xd,rd,yd", [("bf16", None, "bf16"), ("bf16", "bf16", "bf16"), ("fp32", None, "bf16"), ("bf16", "fp32", "fp32")])
@pytest.mark.parametrize("D", WIDTHS)
def test_rows(D, xd, rd, yd):
    base.test_forward_and_backward(2, 150, D, 0, xd, rd, yd)


@pytest.mark.parametrize("xd,rd", [("bf16", None), ("bf16", "bf16"), ("fp32", "fp32")])
@pytest.mark.parametrize("block", [None, 128])
@pytest.mark.parametrize("D", WIDTHS)
def test_8_bits(D, block, xd, rd):
    base.test_8_bit_results(300, D, 0, block, xd, rd)


@pytest.mark.parametrize("xd,yd", [("bf16", "bf16"), ("fp32", "bf16")])
@pytest.mark.parametrize("D", [8, 24, 32, 40, 56, 64, 72, 88, 92, 96, 100, 104, 120, 124, 128])
def test_heads(D, xd, yd):
    base.test_heads_inside_a_packed_projection(150, 7, D, xd, yd)
