"""The sigmoid gate's gradient where the sigmoid is near one: its factor 1 - s_k = 1 / (1 + exp(l_k)) keeps its relative
precision (exp to 2 units, one sum, one division: under 8 half-units), so the bound of w (|g| + sum |g| w) scales with it."""
import pytest
import torch

import layer_util as L

pytestmark = pytest.mark.gpu
U = L.ULP32


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("E,K", [(16, 2), (100, 7), (256, 8), (1024, 16)])
@pytest.mark.parametrize("centre", [-20.0, 0.0, 4.0, 8.0, 10.0, 16.0, 20.0, 40.0])
def test_gradient_of_large_logits(centre, E, K, dtype):
    import paper_2609_36959_b200 as cb
    gen = torch.Generator(device="cuda").manual_seed(E + K)
    T = 203
    logits = (torch.randn((T, E), generator=gen, device="cuda") + centre).to(dtype)
    g = torch.randn((T, K), generator=gen, device="cuda")
    ids, w = torch.empty((T, K), dtype=torch.int32, device="cuda"), torch.empty((T, K), device="cuda")
    grad = torch.full_like(logits, 7.0)
    cb.gate_topk(logits, ids, w, flags=cb.GATE_SIGMOID)
    cb.gate_topk_backward(g, logits, ids, w, grad, flags=cb.GATE_SIGMOID)
    torch.cuda.synchronize()
    assert cb.read_and_clear_device_error() == 0
    at = ids.long()
    ref = L.gate_backward(g, logits, at, w, True)
    wd, gd = w.double(), g.double().abs()
    terms = wd * (gd + (gd * wd).sum(1, keepdim=True)) * torch.sigmoid(-logits.double().gather(1, at))
    bound = torch.zeros_like(ref).scatter_(1, at, 64 * U * terms)
    half = 2 * L.ULP16 if dtype == torch.bfloat16 else 2 * U
    assert ((grad.double() - ref).abs() <= bound + half * ref.abs() + 1e-38).all()


def test_masked_and_infinite_logits():
    """Weights of 0 keep gradients of 0, and a chosen +inf has the factor 0."""
    import math

    import paper_2609_36959_b200 as cb
    logits = torch.full((3, 8), -math.inf, device="cuda")
    logits[1, 5] = 3.0
    logits[2, 2], logits[2, 6] = math.inf, 1.0
    ids, w, grad = torch.empty((3, 4), dtype=torch.int32, device="cuda"), torch.empty((3, 4), device="cuda"), torch.full_like(logits, 7.0)
    g = torch.tensor([[1.0, 2.0, 3.0, 4.0]], device="cuda").repeat(3, 1)
    cb.gate_topk(logits, ids, w, flags=cb.GATE_SIGMOID)
    cb.gate_topk_backward(g, logits, ids, w, grad, flags=cb.GATE_SIGMOID)
    torch.cuda.synchronize()
    assert ids[2, :2].tolist() == [2, 6] and float(grad[0].abs().sum()) == 0 and float(grad[1].abs().sum()) == 0
    assert float(grad[2, 2]) == 0 and bool(torch.isfinite(grad[2]).all()) and float(grad[2, 6]) != 0
