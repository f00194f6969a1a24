"""32-bit rows whose sum is not exact: a constant row has z = 0 exactly and its own value as the mean, and rows with a
spread far below their mean keep it.

A first mean is off by up to 64 u |x| (u = 2^-24); the mean of the differences from it corrects that up to the rounding of
the result, u |x|, and the differences' own sum, 64 u times 64 u |x|.  So z is off by rstd (2 u |x|) where the values
themselves are given to u |x|, and by 64 u (|z| + rstd mean|x - mean|) as of any other sum."""
import pytest
import torch

import layer_util as L

pytestmark = pytest.mark.gpu
U = L.ULP32
# one warp a row, a CTA a row (of two and four vectors a thread), and the rings (four rows, one row, two and four vectors)
SHAPES = [(5, 24), (700, 264), (40, 1000), (3, 1024), (20, 1640), (7, 5000), (3, 16384), (2371, 2056), (1201, 4096), (611, 6144), (611, 16384)]


def _forward(x, gamma, beta, eps):
    import paper_2609_36959_b200 as cb
    y, mean, rstd = torch.full_like(x, 7.0), torch.full((x.shape[0],), 7.0, device="cuda"), torch.full((x.shape[0],), 7.0, device="cuda")
    cb.layer_norm(x, gamma, beta, eps, y, mean, rstd)
    torch.cuda.synchronize()
    return y, mean, rstd


@pytest.mark.parametrize("T,H", SHAPES)
def test_constant_rows_are_exact(T, H):
    gamma, beta = torch.rand(H, device="cuda") + 0.5, torch.randn(H, device="cuda")
    values = torch.tensor([1000.1, 10000.1, -3.3e-5, 0.1, -7.7e8, 1e-30, 3.1e30], device="cuda")
    c = values[torch.arange(T, device="cuda") % 7]
    x = c[:, None].expand(T, H).contiguous()
    y, mean, rstd = _forward(x, gamma, beta, 1e-5)
    assert torch.equal(mean, c)
    assert torch.equal(y, beta.expand(T, H))
    usual = c.abs() < 1e9          # (the squares of larger differences overflow: those rows have rstd = 0)
    assert ((rstd[usual].double() - 1e5 ** 0.5).abs() <= 1e-4 * 1e5 ** 0.5).all()


@pytest.mark.parametrize("T,H", SHAPES)
def test_small_spread_about_a_large_mean(T, H):
    g = torch.Generator(device="cuda").manual_seed(H)
    x = 10000.1 + 0.05 * torch.randn((T, H), generator=g, device="cuda")
    gamma, beta = torch.ones(H, device="cuda"), torch.zeros(H, device="cuda")
    y, mean, rstd = _forward(x, gamma, beta, 1e-5)
    _, mu, rs, z = L.norm_forward(x, gamma, beta, 1e-5)
    ax = x.double().abs()
    spread = (x.double() - mu).abs().mean(1, keepdim=True)
    off = rs * 2 * U * ax + 64 * U * (z.abs() + rs * spread)
    assert ((mean[:, None].double() - mu).abs() <= 2 * U * ax + 64 * U * spread).all()
    # the variance about a mean that is off by m is off by m^2, far below; its own sum by 64 u
    assert ((rstd[:, None].double() - rs).abs() <= rs * 128 * U).all()
    assert ((y.double() - z).abs() <= off + z.abs() * 128 * U).all()


def test_not_finite_rows_stay_so():
    H = 1000
    x = torch.randn((6, H), device="cuda")
    x[1, 3], x[2, 4], x[3, 5] = float("nan"), float("inf"), float("-inf")
    y, mean, rstd = _forward(x, torch.ones(H, device="cuda"), torch.zeros(H, device="cuda"), 1e-5)
    assert torch.isnan(y).all(1).tolist() == [False, True, True, True, False, False]
    assert torch.isfinite(rstd).tolist() == [True, False, False, False, True, True]
