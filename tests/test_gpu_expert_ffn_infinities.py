"""Pre-activations that are infinite: the saved codes keep them, so the gradients are as little finite as the formula's.
Codes: sign, six exponent and nine mantissa bits; the largest exponent with mantissa 0 is an infinity, with another a NaN."""
import pytest
import torch

import layer_util as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("P", [4, 90])                            # a few rows, and tiles
def test_infinite_preactivations(P):
    import paper_2609_36959_b200 as cb
    H = F = 16
    g = torch.Generator(device="cuda").manual_seed(P)

    def rnd(*s):
        return torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)

    rows, dy, wgu, wd = rnd(P, H), rnd(P, H), rnd(1, 2 * F, H), rnd(1, H, F)
    inf = float("inf")
    rows[1, 3], rows[3, 5] = inf, -inf                            # one infinite product a sum: no NaN before the activation
    off = torch.tensor([0, P], dtype=torch.int32, device="cuda")
    slot = torch.zeros(1, dtype=torch.int32, device="cuda")
    act, out, pre, dpre, dx = (torch.full((P, n), 7.0, dtype=torch.bfloat16, device="cuda") for n in (F, H, 2 * F, 2 * F, H))
    ws = torch.empty(cb.expert_ffn_workspace_bytes(P, 1, 1, H, F), dtype=torch.uint8, device="cuda")
    cb.expert_ffn(rows, off, slot, wgu, wd, act, out, ws, pre=pre)
    cb.expert_ffn_backward(dy, rows, off, slot, wgu, wd, pre, act, dpre, ws, grad_rows=dx)
    torch.cuda.synchronize()
    assert cb.read_and_clear_device_error() == 0
    b = L.ffn_backward(dy, rows, [(0, P, 0)], wgu, wd)
    codes = pre.view(torch.int16).to(torch.int64) & 0xFFFF
    want = b["pre"]
    assert torch.equal(codes == 0x7E00, want == inf) and torch.equal(codes == 0xFE00, want == -inf)
    assert int((want.abs() == inf).sum()) == 4 * F
    for name, got in (("d_pre", dpre), ("dx", dx)):
        assert torch.equal(torch.isfinite(got.float()), torch.isfinite(b[name])), name
