"""The norm's forms for many rows of 129 to 896 vectors (four vectors a thread) and gamma on a 16-byte boundary that is none of 32, against
the 64-bit form.  Bounds as in the general tests (u = 2^-24): rstd 24 u, y 26 u and half a step of its type, codes half a step of theirs
and 64 u; gamma's gradient an fp32 sum over the rows."""
import pytest
import torch

import dense_util as D

pytestmark = pytest.mark.gpu
U, BF16 = D.U, torch.bfloat16


def _inputs(T, H, dtype, seed, shift):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, r, dy = (torch.randn((T, H), generator=g, device="cuda").to(dtype) for _ in range(3))
    room = torch.randn(H + 16, generator=g, device="cuda") * 0.3 + 1
    gamma = room[shift:shift + H]
    assert gamma.data_ptr() % 32 == 4 * shift % 32 and gamma.data_ptr() % 16 == 0
    return x, r, dy, gamma


def _y_is_right(y, ref, dtype):
    return ((y.double() - ref).abs() <= (26 * U + D.HALF[dtype]) * (1 + 32 * U) * ref.abs() + 1e-38).all()


@pytest.mark.parametrize("shift", [0, 4])
@pytest.mark.parametrize("dtype,T,H", [(BF16, 16300, 1032), (BF16, 8300, 2048), (BF16, 1100, 4096), (BF16, 600, 7168), (torch.float32, 16300, 520),
                                       (torch.float32, 8300, 1024), (torch.float32, 600, 3584)])
def test_norm_of_many_rows(dtype, T, H, shift):
    import paper_2609_36959_b200 as cb
    x, r, dy, gamma = _inputs(T, H, dtype, T + H, shift)
    total, y = torch.empty_like(x), torch.full((T + 1, H), 7.0, dtype=dtype, device="cuda")
    rstd = torch.empty(T, device="cuda")
    cb.rms_norm(x, gamma, 1e-5, residual=r, sum_out=total, y=y[:T], rstd=rstd)
    assert torch.equal(total, (x.double() + r.double()).to(dtype)) and (y[T] == 7).all()
    ref, rs = D.rms_forward(total, gamma, 1e-5)
    assert ((rstd.double() - rs[:, 0]).abs() <= 24 * U * rs[:, 0]).all() and _y_is_right(y[:T], ref, dtype)
    for code, group in ((torch.float8_e4m3fn, 0), (torch.float8_e4m3fn, 128), (torch.int8, 0), (torch.int8, 128)):
        q = torch.full((T + 1, H), 7, dtype=torch.uint8, device="cuda").view(code)
        scales = torch.full((T + 1, len(D.groups_of(H, group))), 7.0, device="cuda")
        cb.rms_norm(x, gamma, 1e-5, residual=r, y=y[:T], packed=(q[:T], scales[:T]))
        assert (q[T].view(torch.uint8) == 7).all() and (scales[T] == 7).all() and _y_is_right(y[:T], ref, dtype)
        got, step = D.values(q[:T], scales[:T], group), D.values(torch.ones_like(ref), scales[:T], group)
        tol = (0.5 + 127 * 64 * U) * step if code == torch.int8 else torch.maximum(2.0 ** -4 * (1 + 64 * U) * ref.abs(), 2.0 ** -10 * (1 + 64 * U) * step)
        assert ((got - ref).abs() <= tol + 64 * U * ref.abs()).all()
        most = D.values(torch.ones_like(ref), torch.stack([ref[:, a:b].abs().amax(1) for a, b in D.groups_of(H, group)], 1), group)
        assert ((step * D.LARGEST[code] - most).abs() <= 32 * U * most).all()
    # the gradients, gamma on the same boundary
    dx, dg = torch.empty_like(x), torch.empty(H, device="cuda")
    ws = torch.empty(cb.rms_norm_workspace_bytes(T, H), dtype=torch.uint8, device="cuda")
    cb.rms_norm_backward(dy, total, gamma, rstd, dx, dg, ws)
    rx, rg = D.rms_backward(dy, total, gamma, rstd.double()[:, None])
    z = total.double() * rstd.double()[:, None]
    g = (dy.double() * gamma.double()).abs()
    tol = 64 * U * rstd.double()[:, None] * (g + z.abs() * (g * z.abs()).mean(1, keepdim=True)) + D.HALF[dtype] * rx.abs() * (1 + 64 * U) + 1e-38
    assert ((dx.double() - rx).abs() <= tol).all()
    assert ((dg.double() - rg).abs() <= (T + 68) * U * (dy.double() * z).abs().sum(0) + 1e-38).all()
