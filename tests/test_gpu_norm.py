"""Layer norm and its gradients against the 64-bit plain form.

Bounds (u = 2^-24, half a unit of fp32): a sum of a row is 32 additions in a thread and ten levels of a tree, so the
mean is off by at most 42 u mean|x|, z by 64 u (|z| + rstd (|x| + mean|x|)) with the roundings of the variance and the
products; bf16 results add half a unit of bf16, 2^-9 |result| (taken twice).  The weights' gradients are fp32 sums over T
rows: (T + 64) u sum|dy z| in any order, plus what z is off by."""
import pytest
import torch

import layer_util as L

pytestmark = pytest.mark.gpu
U = L.ULP32


def _run(x, gamma, beta, dy, eps):
    import paper_2609_36959_b200 as cb
    T, H = x.shape
    dev = x.device

    def f32(*s):
        return torch.full(s, 7.0, device=dev)

    y, dx, mean, rstd, dg, db = torch.full_like(x, 7.0), torch.full_like(x, 7.0), f32(T), f32(T), f32(H), f32(H)
    ws = torch.full((cb.layer_norm_workspace_bytes(T, H),), 0xAB, dtype=torch.uint8, device=dev)
    cb.layer_norm(x, gamma, beta, eps, y, mean, rstd)
    cb.layer_norm_backward(dy, x, gamma, mean, rstd, dx, dg, db, ws)
    torch.cuda.synchronize()
    return y, mean, rstd, dx, dg, db


def _check(x, gamma, beta, dy, eps, got):
    y, mean, rstd, dx, dg, db = (t.double() for t in got)
    T, H = x.shape
    half = 2 * L.ULP16 if x.dtype == torch.bfloat16 else 2 * U
    ref, mu, rs, z = L.norm_forward(x, gamma, beta, eps)
    rx, rg, rb = L.norm_backward(dy, x, gamma, eps)
    xd, ga, dyd = x.double(), gamma.double().abs(), dy.double()
    ax = xd.abs().mean(1, keepdim=True)
    dz = 64 * U * (z.abs() + rs * (xd.abs() + ax))
    assert ((mean[:, None] - mu).abs() <= 64 * U * ax + 1e-40).all()
    assert ((y - ref).abs() <= ga * dz + 4 * U * beta.double().abs() + half * ref.abs() + 1e-38).all()
    g = (dyd * gamma.double()).abs()
    c1, c2 = g.mean(1, keepdim=True), (g * z.abs()).mean(1, keepdim=True)
    tol = rs * (64 * U * (g + c1 + z.abs() * c2) + dz * c2 + z.abs() * (g * dz).mean(1, keepdim=True))
    # rstd itself is off by its variance's rounding: relative 64 u (1 + mean (|x| rstd) mean|z|)
    tol = tol + rx.abs() * 64 * U * (1 + rs * ax) + half * rx.abs() + 1e-38
    assert ((dx - rx).abs() <= tol).all(), float(((dx - rx).abs() - tol).max())
    assert ((dg - rg).abs() <= (T + 64) * U * (dyd * z).abs().sum(0) + (dyd.abs() * dz).sum(0) + 1e-38).all()
    assert ((db - rb).abs() <= (T + 64) * U * dyd.abs().sum(0) + 1e-38).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H", [(1, 8), (1, 7168), (3, 24), (5, 256), (700, 264), (33, 512), (9, 1000), (2000, 1024), (17, 1032),
                                 (300, 4096), (5, 8192), (6, 8200), (3, 16384)])
def test_norm_against_plain(T, H, dtype):
    g = torch.Generator(device="cuda").manual_seed(T * 100003 + H)
    x = (torch.randn((T, H), generator=g, device="cuda") * 2 + 0.5).to(dtype)
    dy = torch.randn((T, H), generator=g, device="cuda").to(dtype)
    gamma, beta = torch.randn(H, generator=g, device="cuda") * 0.3 + 1, torch.randn(H, generator=g, device="cuda")
    got = _run(x, gamma, beta, dy, 1e-5)
    _check(x, gamma, beta, dy, 1e-5, got)
    again = _run(x, gamma, beta, dy, 1e-5)
    assert all(torch.equal(a, b) for a, b in zip(got, again))       # the same bits every time


def test_norm_rows_far_from_zero_and_constant_rows():
    """Rows whose mean is a thousand times their spread (a difference of squares would lose the variance), and rows
    without any spread: rstd = 1 / sqrt(eps)."""
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((64, 640), generator=g, device="cuda") + 1000.0
    x[7] = 3.25
    x[8] = 0.0
    dy = torch.randn((64, 640), generator=g, device="cuda")
    gamma, beta = torch.ones(640, device="cuda"), torch.zeros(640, device="cuda")
    got = _run(x, gamma, beta, dy, 1e-5)
    _check(x, gamma, beta, dy, 1e-5, got)
    assert torch.equal(got[0][7], torch.zeros_like(got[0][7])) and abs(float(got[2][8]) - 1e5 ** 0.5) < 1e-3


def test_norm_no_rows_in_place_other_stream_and_nan_stays_in_its_row():
    import paper_2609_36959_b200 as cb
    dev = "cuda"
    H = 1032
    e = torch.empty((0, H), device=dev)
    dg, db = torch.full((H,), 5.0, device=dev), torch.full((H,), 5.0, device=dev)
    ws = torch.empty(cb.layer_norm_workspace_bytes(4096, H), dtype=torch.uint8, device=dev)
    none = torch.empty(0, device=dev)
    gamma, beta = torch.rand(H, device=dev), torch.rand(H, device=dev)
    cb.layer_norm(e, gamma, beta, 1e-5, e, none, none)
    cb.layer_norm_backward(e, e, gamma, none, none, e, dg, db, ws)
    torch.cuda.synchronize()
    assert float(dg.abs().sum()) == 0 and float(db.abs().sum()) == 0
    x = torch.randn((50, H), device=dev).to(torch.bfloat16)
    x[20, 5] = float("nan")
    x[21, 6] = float("inf")
    dy = torch.randn((50, H), device=dev).to(torch.bfloat16)
    got = _run(x, gamma, beta, dy, 1e-5)
    bad = torch.isnan(got[0].float()).any(1)
    assert bad.tolist() == [r in (20, 21) for r in range(50)]
    assert torch.isnan(got[3].float()).any(1).tolist() == bad.tolist()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        xi, dyi, mean, rstd = x.clone(), dy.clone(), torch.empty(50, device=dev), torch.empty(50, device=dev)
        cb.layer_norm_backward(dyi, x, gamma, got[1], got[2], dyi, dg, db, ws)       # grad_x over grad_y
        cb.layer_norm(xi, gamma, beta, 1e-5, xi, mean, rstd)                        # y over x
    side.synchronize()
    assert torch.equal(xi.view(torch.int16), got[0].view(torch.int16))
    assert torch.equal(dyi.view(torch.int16), got[3].view(torch.int16))


def test_norm_gradient_against_differences():
    """Directional derivatives of the 64-bit forward pass against the kernel's fp32 gradients: central differences
    with step 1e-5 are good to 1e-8 of the loss terms' sum, the gradients to the bounds above, 1e-4 in all."""
    g = torch.Generator(device="cuda").manual_seed(9)
    x, dy, v = (torch.randn((11, 72), generator=g, device="cuda") for _ in range(3))
    gamma, beta, vg = (torch.randn(72, generator=g, device="cuda") for _ in range(3))
    _, _, _, dx, dg, _ = _run(x, gamma, beta, dy, 1e-5)

    def loss(xx, gg):
        return float((L.norm_forward(xx, gg, beta, 1e-5)[0] * dy.double()).sum())

    h, xd, gd = 1e-5, x.double(), gamma.double()
    num = (loss(xd + h * v.double(), gd) - loss(xd - h * v.double(), gd)) / (2 * h)
    assert abs(num - float((dx.double() * v.double()).sum())) <= 1e-4 * float((dx.double() * v.double()).abs().sum())
    num = (loss(xd, gd + h * vg.double()) - loss(xd, gd - h * vg.double())) / (2 * h)
    assert abs(num - float((dg.double() * vg.double()).sum())) <= 1e-4 * float((dg.double() * vg.double()).abs().sum())
