"""The norm's ring kernels against the 64-bit plain form: enough rows that every CTA reuses its slots, ragged last groups,
one, two and four vectors a thread, one slot to four.  The bounds are those of the other norm tests.

The forward pass takes the ring from four turns a CTA on (T >= 4 x rows of a slot x CTAs): with 148 SMs that is 4736 rows up
to 512 vectors a row, 2368 up to 896, and 1184 or 592 above, with one or two CTAs an SM; more SMs leave some shapes to the
other kernels.  The backward pass takes it for every row of more than 128 vectors."""
import pytest
import torch

from test_gpu_norm import _check, _run

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
SHAPES = [(4739, 4096, BF16), (2371, 7168, BF16), (1203, 8192, BF16), (611, 12288, BF16), (1203, 16384, BF16),
          (4739, 1032, F32), (2371, 2056, F32), (1201, 4096, F32), (611, 6144, F32), (1203, 8192, F32), (611, 16384, F32)]


def _inputs(T, H, dtype):
    g = torch.Generator(device="cuda").manual_seed(T + H)
    x = (torch.randn((T, H), generator=g, device="cuda") * 2 + 0.5).to(dtype)
    dy = torch.randn((T, H), generator=g, device="cuda").to(dtype)
    gamma, beta = torch.randn(H, generator=g, device="cuda") * 0.3 + 1, torch.randn(H, generator=g, device="cuda")
    return x, gamma, beta, dy


@pytest.mark.parametrize("T,H,dtype", SHAPES)
def test_rings_against_plain(T, H, dtype):
    import paper_2609_36959_b200 as cb
    x, gamma, beta, dy = _inputs(T, H, dtype)
    got = _run(x, gamma, beta, dy, 1e-5)
    assert cb.read_and_clear_device_error() == 0
    _check(x, gamma, beta, dy, 1e-5, got)
    again = _run(x, gamma, beta, dy, 1e-5)
    assert all(torch.equal(a, b) for a, b in zip(got, again))       # the same bits every time
    # rows do not depend on their neighbours or on the kernel form beyond the order of a sum: a few rows alone agree
    few = _run(x[-3:].contiguous(), gamma, beta, dy[-3:].contiguous(), 1e-5)
    _check(x[-3:], gamma, beta, dy[-3:], 1e-5, few)


@pytest.mark.parametrize("T,H,dtype", SHAPES)
def test_rings_in_place(T, H, dtype):
    import paper_2609_36959_b200 as cb
    x, gamma, beta, dy = _inputs(T, H, dtype)
    y, mean, rstd, dx, dg, db = _run(x, gamma, beta, dy, 1e-5)
    ws = torch.empty(cb.layer_norm_workspace_bytes(T, H), dtype=torch.uint8, device="cuda")
    dg2, db2, mean2, rstd2 = (torch.empty_like(t) for t in (dg, db, mean, rstd))
    cb.layer_norm_backward(dy, x, gamma, mean, rstd, dy, dg2, db2, ws)
    cb.layer_norm(x, gamma, beta, 1e-5, x, mean2, rstd2)
    torch.cuda.synchronize()
    for a, b in ((y, x), (dx, dy), (dg, dg2), (db, db2), (mean, mean2), (rstd, rstd2)):
        assert torch.equal(a, b)


def test_not_finite_rows_stay_in_their_row():
    T, H = 2371, 7168
    x, gamma, beta, dy = _inputs(T, H, BF16)
    clean = _run(x, gamma, beta, dy, 1e-5)
    bad = [0, 5, 295, 296, 1001, T - 1]
    x[bad[::2], 7], x[bad[1::2], H - 1] = float("nan"), float("inf")
    got = _run(x, gamma, beta, dy, 1e-5)
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[bad] = False
    for k in (0, 3):                                                # y, dx
        assert torch.equal(got[k][keep], clean[k][keep])
        assert bool(torch.isnan(got[k][~keep].float()).all())
