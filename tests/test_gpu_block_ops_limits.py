"""Block operators at the limits of their ranges: gates far out, more column tiles than a grid dimension holds, results given by
the caller."""
import numpy as np
import pytest
import torch

from oracle import block_ops as ob

pytestmark = pytest.mark.gpu

DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_gradients_of_gates_far_out(act, dt):
    # where the activation is g or 0 its slope is 1 or 0 exactly, up to the largest gates (the square of 2e19 is past fp32)
    import paper_2511_20390_b200 as free
    far = [120.0, 1e4, 1e10, 1.5e19, 2e19, 1e25, 1e30, 3e38]
    gates = torch.tensor([-v for v in far[::-1]] + far, device="cuda").to(DT[dt])
    M, F, K, step = 5, len(gates), 8, 2.0 ** -10
    pre = torch.cat([gates, torch.ones_like(gates)]).repeat(M, 1)
    x, w = torch.ones(M, K, dtype=DT[dt], device="cuda"), torch.zeros(2 * F, K, dtype=DT[dt], device="cuda")
    w[0] = 1.0                                                     # its slope is 0, so dx is 0
    dh = torch.full((M, F), step, dtype=DT[dt], device="cuda")
    dx, dw, db = free.op_gated_linear_bwd(x, w, pre, dh, act=act)
    slope = np.concatenate([np.zeros(F // 2), np.ones(F // 2)])
    assert not np.any(ob.gate_act(act, np.array([-700.0]))[1] > 1e-300) and ob.gate_act(act, np.array([700.0]))[1] == 1.0
    assert np.array_equal(db[:F].cpu().numpy(), M * step * slope)
    assert np.array_equal(dw[:F].double().cpu().numpy(), np.repeat((M * step * slope)[:, None], K, 1))
    # five equal terms, each rounded once, and four sums: 2^-21 of them; dw is rounded to its type besides
    a = gates.double().cpu().numpy() * slope
    assert (np.abs(db[F:].double().cpu().numpy() - M * step * a) <= 2.0 ** -21 * M * step * a).all()
    half = torch.finfo(DT[dt]).eps / 2
    assert (np.abs(dw[F:].double().cpu().numpy() - (M * step * a)[:, None]) <= (2.0 ** -21 + half) * (M * step * a)[:, None]).all()
    assert not dx.any() and not torch.isnan(dx).any()
