"""The gate against the 64-bit plain form: ids equal, weights within 64 fp32 half-units of the value (exp and the
division are good to a few units, the sum of up to 16 positive terms to 16), gradients within 64 half-units of
w (|g| + sum |g| w), which the subtraction may cancel; bf16 gradients add half a unit of bf16 (taken twice)."""
import math

import pytest
import torch

import layer_util as L

pytestmark = pytest.mark.gpu
U = L.ULP32


def _run(logits, K, sigmoid, g=None):
    import paper_2609_36959_b200 as cb
    T, E = logits.shape
    flags = cb.GATE_SIGMOID if sigmoid else 0
    ids = torch.full((T, K), -9, dtype=torch.int32, device="cuda")
    w = torch.full((T, K), 7.0, device="cuda")
    cb.gate_topk(logits, ids, w, flags=flags)
    grad = None
    if g is not None:
        grad = torch.full_like(logits, 7.0)
        cb.gate_topk_backward(g, logits, ids, w, grad, flags=flags)
    torch.cuda.synchronize()
    assert cb.read_and_clear_device_error() == 0
    return ids, w, grad


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,E,K", [(1, 1, 1), (1, 8, 8), (3, 16, 16), (257, 16, 2), (100, 17, 5), (9, 33, 1), (1000, 64, 6), (77, 100, 7),
                                   (513, 128, 8), (40, 250, 9), (4099, 256, 8), (31, 384, 12), (65, 512, 3), (29, 1000, 15), (50, 1024, 16)])
def test_gate_against_plain(T, E, K, dtype, sigmoid):
    gen = torch.Generator(device="cuda").manual_seed(T + 7 * E + K)
    logits = (torch.randn((T, E), generator=gen, device="cuda") * 3).to(dtype)
    g = torch.randn((T, K), generator=gen, device="cuda")
    ids, w, grad = _run(logits, K, sigmoid, g)
    rid, rw, _ = L.gate_forward(logits, K, sigmoid)
    assert torch.equal(ids.long(), rid)
    assert ((w.double() - rw).abs() <= 64 * U * rw + 1e-38).all()
    # the backward pass of the weights that the forward pass gave
    ref = L.gate_backward(g, logits, rid, w, sigmoid)
    gw = (g.double().abs() * w.double()).sum(1, keepdim=True)
    bound = torch.zeros_like(ref).scatter_(1, rid, 64 * U * w.double() * (g.double().abs() + gw))
    half = 2 * L.ULP16 if dtype == torch.bfloat16 else 2 * U
    assert ((grad.double() - ref).abs() <= bound + half * ref.abs() + 1e-38).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gate_ties_masks_and_non_finite_logits(dtype):
    E, K = 40, 4
    low = torch.finfo(dtype).min
    rows = torch.zeros((10, E), dtype=dtype)
    rows[1, 20:] = 1.0                                   # ties: ids 20..23
    rows[2, ::2] = -0.0                                  # -0 equals +0: ids 0..3
    rows[3] = -math.inf                                  # nothing left: ids 0..3, weights 0
    rows[4] = -math.inf
    rows[4, 35], rows[4, 7] = 2.0, 2.0                   # two left of four wanted
    rows[5] = low                                        # everything at the type's lowest value: equal weights
    rows[6] = low
    rows[6, 39] = 0.0
    rows[7, 11] = math.nan                               # chosen first, shows in the weights
    rows[8] = -80.0                                      # sigmoids far below one
    rows[8, 3] = -79.0
    rows[9] = -200.0                                     # sigmoids that underflow in fp32
    rows[9, 5] = -199.0
    rows = rows.cuda()
    for sigmoid in (False, True):
        ids, w, grad = _run(rows, K, sigmoid, torch.ones((10, K), device="cuda"))
        rid, rw, _ = L.gate_forward(rows, K, sigmoid)
        assert torch.equal(ids.long(), rid)
        assert ids.tolist()[0] == [0, 1, 2, 3] and ids.tolist()[1] == [20, 21, 22, 23] and ids.tolist()[2] == [0, 1, 2, 3]
        assert ids.tolist()[3] == [0, 1, 2, 3] and w[3].tolist() == [0.0] * 4 and float(grad[3].abs().sum()) == 0
        assert ids.tolist()[4] == [7, 35, 0, 1] and w[4].tolist() == [0.5, 0.5, 0.0, 0.0]
        assert w[5].tolist() == [0.25] * 4 and ids.tolist()[6][0] == 39 and w[6].tolist() == [1.0, 0.0, 0.0, 0.0]
        assert ids.tolist()[7][0] == 11 and bool(torch.isnan(w[7]).all())
        keep = [r for r in range(10) if r != 7]
        assert ((w.double() - rw)[keep].abs() <= 64 * U * rw[keep] + 1e-38).all()
        assert bool(torch.isfinite(grad[keep].float()).all())


def test_gate_bad_ids_are_flagged_and_skipped():
    import paper_2609_36959_b200 as cb
    ids = torch.tensor([[0, 99], [-1, 2]], dtype=torch.int32, device="cuda")
    w, g = torch.full((2, 2), 0.5, device="cuda"), torch.tensor([[1.0, 2.0], [3.0, 5.0]], device="cuda")
    grad = torch.full((2, 8), 7.0, device="cuda")
    cb.gate_topk_backward(g, torch.zeros((2, 8), device="cuda"), ids, w, grad)
    torch.cuda.synchronize()
    assert cb.read_and_clear_device_error() == cb.DEVERR_BAD_EXPERT_ID
    want = torch.zeros((2, 8))
    want[0, 0], want[1, 2] = 0.5 * (1.0 - 1.5), 0.5 * (5.0 - 4.0)
    assert torch.equal(grad.cpu(), want)


def test_gate_gradient_against_differences():
    gen = torch.Generator(device="cuda").manual_seed(2)
    logits, v = (torch.randn((23, 30), generator=gen, device="cuda") * 2 for _ in range(2))
    g = torch.randn((23, 5), generator=gen, device="cuda")
    for sigmoid in (False, True):
        ids, _, grad = _run(logits, 5, sigmoid, g)

        def loss(t):             # the choice itself is held fixed: its derivative is 0 almost everywhere
            return float((L.gate_weights(t.gather(1, ids.long()), sigmoid) * g.double()).sum())

        h = 1e-6
        num = (loss(logits.double() + h * v.double()) - loss(logits.double() - h * v.double())) / (2 * h)
        terms = (grad.double() * v.double())
        assert abs(num - float(terms.sum())) <= 1e-4 * float(terms.abs().sum())
