"""The layer's buffers under calls that come twice or feed a call's own result back."""
import pytest
import torch

import workloads as W
from test_gpu_moe_layer import _layer

pytestmark = pytest.mark.gpu
GRADS = ("grad_gamma", "grad_beta", "grad_w_router", "grad_w_gate_up", "grad_w_down")


def _bits(t):
    return t.clone().view(torch.uint8)


@pytest.mark.parametrize("T", [3, 60])
def test_backward_twice_gives_the_same(T):
    w = W.make_custom(T, 8, 2, 64, 2, 2, 3, seed=3, C=2)
    m, x, dy = _layer(w, 40, "sigmoid", 0.2)
    m.forward(x, 5)
    first = [_bits(m.backward(dy))] + [_bits(getattr(m, g)) for g in GRADS]
    other = m.backward(-2 * dy)                                   # another gradient of the same forward call in between
    assert bool(torch.isfinite(other.float()).all())
    again = [_bits(m.backward(dy))] + [_bits(getattr(m, g)) for g in GRADS]
    for a, b in zip(first, again):
        assert torch.equal(a, b)


def test_gradient_fed_back_is_read_before_it_is_overwritten():
    w = W.make_custom(60, 8, 2, 64, 2, 2, 3, seed=3, C=2)
    m, x, dy = _layer(w, 40, "softmax", 0.2)
    m.forward(x, 5)
    g = m.backward(dy)
    kept = g.clone()
    want = _bits(m.backward(kept))
    g = m.backward(dy)
    assert torch.equal(_bits(m.backward(g)), want)                # g is the buffer that the call writes


def test_output_fed_back_can_not_be_differentiated():
    import paper_2609_36959_b200 as cb
    w = W.make_custom(60, 8, 2, 64, 2, 2, 3, seed=3, C=2)
    m, x, dy = _layer(w, 40, "softmax", 0.2)
    want = _bits(m.forward(m.forward(x, 5).clone(), 6))
    assert torch.equal(_bits(m.forward(m.forward(x, 5), 6)), want)
    with pytest.raises(cb.CobaltError):                           # its input was overwritten by its output
        m.backward(dy)
    m.forward(x, 5)
    m.backward(dy)


def test_backward_without_forward_is_refused():
    import paper_2609_36959_b200 as cb
    w = W.make_custom(20, 8, 2, 64, 2, 2, 3, seed=3, C=2)
    m, _, dy = _layer(w, 40, "softmax", 0.2)
    with pytest.raises(cb.CobaltError):
        m.backward(dy)


def test_no_tokens():
    import paper_2609_36959_b200 as cb
    w = W.make_custom(0, 8, 2, 64, 2, 2, 3, seed=3, C=2)
    m, x, dy = _layer(w, 40, "softmax", 0.2)
    assert m.forward(x, 5).shape == (0, 64) and m.backward(dy).shape == (0, 64)
    torch.cuda.synchronize()
    assert cb.read_and_clear_device_error() == 0
    for g in GRADS:
        assert float(getattr(m, g).float().abs().sum()) == 0
