"""The root-mean-square norm at the ends of its range: rows whose sum of squares just fits fp32 and just does not, and rows whose squares vanish."""
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D,fits,not_any_more", [(8192, 2.0e17, 2.1e17), (1152, 5.3e17, 5.6e17), (384, 9.2e17, 9.7e17), (300, 1.0e18, 1.1e18), (64, 2.25e18, 2.4e18), (33, 3.1e18, 3.3e18)])
def test_large_rows(D, fits, not_any_more, dt):
    import paper_2511_20390_b200 as free
    sign = 1 - 2 * (torch.arange(D, device="cuda") % 3 == 0).float()
    x = torch.stack([fits * sign, not_any_more * sign, sign]).to(dt)
    assert (x[0].double() ** 2).sum() < 3.4e38 < (x[1].double() ** 2).sum()
    w = 1 + torch.arange(D, device="cuda") / D
    y, _, _, r = free.op_rms_norm(x, w, out_dtype=torch.float32, want_rstd=True)
    # squares in fp32 (half a step each), their sum in any order, a root of 2 units and two products
    want = x.double() / (x.double() ** 2).mean(1, keepdim=True).sqrt()
    for i in (0, 2):
        assert ((y[i].double() - want[i] * w.double()).abs() <= ((D + 16) * U * want[i] * w.double()).abs()).all()
    assert r[1] == 0 and (y[1] == 0).all()
    # 8 bits: a scale for the row
    q, s, _, _ = free.op_rms_norm(x, out_dtype=torch.float8_e4m3fn)
    back = q.double() * s.double()
    for i in (0, 2):
        assert ((back[i] - want[i]).abs() <= (2.0 ** -4 + (D + 32) * U) * want[i].abs()).all()
    assert (back[1] == 0).all()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D", [8192, 1152, 72, 33])
def test_rows_whose_squares_vanish(D, dt):
    """Magnitudes of 1e-30: the mean square is 0 beside eps, and y = x / sqrt(eps); 8-bit results have a scale of their own still."""
    import paper_2511_20390_b200 as free
    x = (1e-30 * (1 + torch.arange(D, device="cuda") % 7))[None].to(dt)
    y, _, _, r = free.op_rms_norm(x, eps=1e-6, out_dtype=torch.float32, want_rstd=True)
    want = x.double() * 1e3
    assert abs(r.item() - 1e3) <= 8 * U * 1e3
    assert ((y.double() - want).abs() <= 16 * U * want).all()
    q, s, _, _ = free.op_rms_norm(x, eps=1e-6, out_dtype=torch.float8_e4m3fn)
    assert ((q.double() * s.double() - want).abs() <= (2.0 ** -4 + 32 * U) * want).all() and q.float().max() == 448
