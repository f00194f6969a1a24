"""The operators on token rows where elements lie beyond 2^31 and 2^32: the last rows and some in between, against calls on those rows
alone (or the 64-bit form)."""
import pytest
import torch

import dense_util as D

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
T, H = 270001, 16384                     # 4.4e9 elements
PROBE = [0, 131071, 131072, 262143, 262144, 270000]


def _rows(seed):
    """Rows that repeat every 4099, so that any misplaced one is another row."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    few = torch.randn((4099, H), generator=g, device="cuda").to(BF16)
    x = torch.empty((T, H), dtype=BF16, device="cuda")
    for a in range(0, T, 4099):
        x[a:a + 4099] = few[:min(4099, T - a)]
    return x


@pytest.mark.parametrize("group", [0, 128])
def test_pack_large(group):
    import paper_2609_36959_b200 as cb
    x = _rows(1)
    q, scales = torch.empty((T, H), dtype=torch.int8, device="cuda"), torch.empty((T, H // 128 if group else 1), device="cuda")
    cb.pack_rows(x, q, scales)
    some, some_scales = torch.empty((len(PROBE), H), dtype=torch.int8, device="cuda"), torch.empty((len(PROBE), scales.shape[1]), device="cuda")
    cb.pack_rows(x[PROBE], some, some_scales)
    assert torch.equal(q[PROBE], some) and torch.equal(scales[PROBE], some_scales)
    want = torch.empty((len(PROBE), H), dtype=BF16, device="cuda")
    cb.unpack_rows(some, some_scales, want)
    cb.unpack_rows(q, scales, x)
    assert torch.equal(x[PROBE], want)


def test_rms_norm_large():
    import paper_2609_36959_b200 as cb
    x = _rows(2)
    gamma, rstd, y = torch.randn(H, device="cuda"), torch.empty(T, device="cuda"), torch.empty_like(x)
    cb.rms_norm(x, gamma, 1e-5, y=y, rstd=rstd)
    ref, rs = D.rms_forward(x[PROBE], gamma, 1e-5)
    assert ((y[PROBE].double() - ref).abs() <= (2.0 ** -8 + 32 * D.U) * ref.abs() + 1e-38).all()
    q, scales = torch.empty((T, H), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty((T, 1), device="cuda")
    cb.rms_norm(x, gamma, 1e-5, packed=(q, scales))
    got = D.values(q[PROBE], scales[PROBE], 0)
    assert ((got - ref).abs() <= 2.0 ** -4 * 1.001 * ref.abs() + 2.0 ** -10 * 1.001 * scales[PROBE].double()).all()
    dg, ws = torch.empty(H, device="cuda"), torch.empty(cb.rms_norm_workspace_bytes(T, H), dtype=torch.uint8, device="cuda")
    dy = x.roll(1, 0)
    cb.rms_norm_backward(dy, x, gamma, rstd, y, dg, ws, grad_sum=dy)
    want, _ = D.rms_backward(dy[PROBE], x[PROBE], gamma, rstd[PROBE].double()[:, None], dy[PROBE])
    z = x[PROBE].double() * rstd[PROBE].double()[:, None]
    g = (dy[PROBE].double() * gamma.double()).abs()
    tol = 64 * D.U * rstd[PROBE].double()[:, None] * (g + z.abs() * (g * z.abs()).mean(1, keepdim=True)) + 2.0 ** -8 * 1.001 * want.abs()
    assert ((y[PROBE].double() - want).abs() <= tol + 4 * D.U * dy[PROBE].double().abs() + 1e-38).all()


def test_linear_large():
    """out and the pass over its gradient past 2^32 elements; dx past 2^32 elements, in both forms."""
    import paper_2609_36959_b200 as cb
    K, N = 64, H
    g = torch.Generator(device="cuda").manual_seed(3)
    x, w = torch.randn((T, K), generator=g, device="cuda").to(BF16), (torch.randn((N, K), generator=g, device="cuda") / 8).to(BF16)
    ws = torch.empty(max(cb.linear_workspace_bytes(T, K, N), cb.linear_workspace_bytes(T, N, K), cb.linear_workspace_bytes(T, N, 264)),
                     dtype=torch.uint8, device="cuda")
    out, pre = torch.empty((T, N), dtype=BF16, device="cuda"), (torch.empty((T, N), dtype=torch.int8, device="cuda"), torch.empty((T, N // 128), device="cuda"))
    cb.linear(x, w, out, ws, act="silu", pre=pre)
    ref = D.act(x[PROBE].double() @ w.double().t(), "silu")
    assert ((out[PROBE].double() - ref).abs() <= 2.0 ** -8 * 1.01 * ref.abs() + 2.0 ** -16).all()
    del out
    dy = _rows(4)
    d, gb = torch.empty_like(dy), torch.empty(N, dtype=BF16, device="cuda")
    gx = torch.empty((T, K), dtype=BF16, device="cuda")
    cb.linear_backward(dy, None, w, ws, act="silu", pre=pre, grad_pre=d, grad_x=gx, grad_bias=gb)
    saved = D.values(pre[0][PROBE], pre[1][PROBE], 128)
    want = dy[PROBE].double() * D.act_slope(saved, "silu")
    assert ((d[PROBE].double() - want).abs() <= 2.0 ** -8 * 1.01 * want.abs() + 2.0 ** -16).all()
    ref = d[PROBE].double() @ w.double()
    assert ((gx[PROBE].double() - ref).abs() <= 2.0 ** -8 * 1.01 * ref.abs() + 2 * N * D.U * (d[PROBE].double().abs() @ w.double().abs())).all()
    del pre, d
    for features in (64, 264):                                       # the gradient's rows stay, or stream
        grad, wide = dy[:, :features].contiguous(), (torch.randn((features, H), generator=g, device="cuda") / 8).to(BF16)
        dx = torch.empty((T, H), dtype=BF16, device="cuda")
        cb.linear_backward(grad, None, wide, ws, grad_x=dx)
        ref = grad[PROBE].double() @ wide.double()
        size = 2 * features * D.U * (grad[PROBE].double().abs() @ wide.double().abs())
        assert ((dx[PROBE].double() - ref).abs() <= size + 2.0 ** -8 * 1.01 * ref.abs()).all()
    assert cb.read_and_clear_device_error() == 0
