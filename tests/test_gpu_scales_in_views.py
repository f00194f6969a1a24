"""Rows in 8 bits that start at any token of a longer tensor: their scales then lie on a 4-byte boundary, codes on one of 16 bytes."""
import pytest
import torch

import dense_util as D

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def _packed(T, H, code, group, seed):
    import paper_2609_36959_b200 as cb
    x = torch.randn((T, H), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(BF16)
    q, scales = torch.empty((T, H), dtype=code, device="cuda"), torch.empty((T, len(D.groups_of(H, group))), device="cuda")
    cb.pack_rows(x, q, scales)
    return x, q, scales


@pytest.mark.parametrize("start,T,form", [(1, 1, "plain"), (3, 4, "plain"), (5, 70, "plain"), (7, 300, "residual"), (2, 300, "f32"), (9, 300, "pre")])
def test_linear_of_rows_from_any_token_on(start, T, form):
    import paper_2609_36959_b200 as cb
    K, N = 272, 264
    _, q, scales = _packed(T + 10, K, torch.float8_e4m3fn, 0, 1)
    _, wq, ws = _packed(N, K, torch.float8_e4m3fn, 0, 2)
    room = torch.empty(cb.linear_workspace_bytes(T, K, N), dtype=torch.uint8, device="cuda")
    dtype = torch.float32 if form == "f32" else BF16
    residual = torch.ones((T, N), dtype=dtype, device="cuda") if form == "residual" else None
    pre = torch.empty((T, N), dtype=BF16, device="cuda") if form == "pre" else None
    rows = slice(start, start + T)
    want, got = (torch.empty((T, N), dtype=dtype, device="cuda") for _ in range(2))
    cb.linear((q[rows], scales[rows].clone()), (wq, ws), want, room, residual=residual, pre=pre)
    cb.linear((q[rows], scales[rows]), (wq, ws), got, room, residual=residual, pre=pre)
    assert torch.equal(got, want)
    assert torch.isfinite(got).all()


@pytest.mark.parametrize("H,group", [(272, 0), (272, 128), (4096, 0), (4240, 128)])
@pytest.mark.parametrize("code", [torch.int8, torch.float8_e4m3fn], ids=["i8", "e4m3"])
def test_norm_gradients_of_rows_from_any_token_on(H, group, code):
    import paper_2609_36959_b200 as cb
    T, start = 40, 3
    x, q, scales = _packed(T + 10, H, code, group, 3)
    gamma, rstd = torch.randn(H, device="cuda"), 1 / x.float().square().mean(1).sqrt()
    dy = torch.randn((T, H), device="cuda").to(BF16)
    rows, room = slice(start, start + T), torch.empty(cb.rms_norm_workspace_bytes(T, H), dtype=torch.uint8, device="cuda")
    results = []
    for copy in (torch.Tensor.clone, lambda t: t):
        dx, dg = torch.empty_like(dy), torch.empty(H, device="cuda")
        cb.rms_norm_backward(dy, (q[rows], copy(scales[rows])), gamma, copy(rstd[rows]), dx, dg, room)
        results.append((dx, dg))
    assert all(torch.equal(a, b) for a, b in zip(*results))
    ref, _ = D.rms_backward(dy, D.values(q[rows], scales[rows], group), gamma, rstd[rows].double()[:, None])
    assert float((results[1][0].double() - ref).norm() / ref.norm()) <= D.HALF[BF16]


@pytest.mark.parametrize("H,group", [(272, 0), (272, 128), (4096, 0)])
def test_norm_into_rows_from_any_token_on(H, group):
    import paper_2609_36959_b200 as cb
    T, start = 40, 3
    x, gamma = torch.randn((T, H), device="cuda").to(BF16), torch.randn(H, device="cuda")
    groups = len(D.groups_of(H, group))
    q, scales = torch.full((T + 10, H), 7, dtype=torch.int8, device="cuda"), torch.full((T + 10, groups), 7.0, device="cuda")
    cb.rms_norm(x, gamma, 1e-5, packed=(q[start:start + T], scales[start:start + T]))
    want_q, want_scales = torch.empty((T, H), dtype=torch.int8, device="cuda"), torch.empty((T, groups), device="cuda")
    cb.rms_norm(x, gamma, 1e-5, packed=(want_q, want_scales))
    assert torch.equal(q[start:start + T], want_q) and torch.equal(scales[start:start + T], want_scales)
    for t, rows in ((q, 7), (scales, 7.0)):
        assert (t[:start] == rows).all() and (t[start + T:] == rows).all()
