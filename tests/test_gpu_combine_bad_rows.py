"""Rows outside their range are flagged and count as zero, with the row buffer at the edges of an allocation of its own."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("K", [1, 2, 8, 16])
def test_rows_outside_their_range(K):
    import paper_2609_36959_b200 as cb
    H, P = 1024, 16384                                   # 32 MiB: whole pages, a segment of their own
    T = P // K
    out = torch.randn((P, H), device="cuda").to(torch.bfloat16)
    g = torch.Generator(device="cuda").manual_seed(K)
    row = torch.randint(0, P, (T, K), generator=g, device="cuda", dtype=torch.int32)
    row[0, 0], row[1, -1], row[2, 0], row[3, -1] = -1, P, -2**31, 2**31 - 1
    row[5], row[6, 0], row[7, -1] = -1, 0, P - 1
    w = torch.randn((T, K), generator=g, device="cuda")
    y = torch.full((T, H), 7.0, device="cuda", dtype=torch.bfloat16)
    cb.combine(out, row.reshape(-1), w, y)
    torch.cuda.synchronize()
    assert cb.read_and_clear_device_error() == cb.DEVERR_BAD_SLOT
    ok = (row >= 0) & (row < P)
    terms = torch.where(ok[..., None], out[row.clamp(0, P - 1).long()].double() * w.double()[..., None], torch.zeros((), device="cuda", dtype=torch.float64))
    want = terms.sum(1)
    # K products and sums in fp32, one rounding to bf16 (half a unit, 2^-9), each taken twice
    assert ((y.double() - want).abs() <= 2 * (2.0**-9 * want.abs() + (K + 1) * 2.0**-24 * terms.abs().sum(1))).all()
    assert bool((y[5] == 0).all())
