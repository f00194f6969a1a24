"""Calls without rows: torch tensors without elements have no address, so every row pointer may be NULL."""
import pytest


@pytest.fixture(scope="module")
def cb():
    from paper_2609_36959_b200 import build
    build.build()
    import paper_2609_36959_b200.binding as binding
    return binding


def test_combine_backward_without_tokens(cb):
    def call(T, go=None, gw=None):
        return cb._lib.cobalt_combine_backward(None, None, None, None, T, 2, 64, go, gw, 0, None)

    assert call(0) == call(0, go=16) == cb.OK
    assert call(4) == call(4, go=16) == cb.ERR_INVALID_ARG


def test_other_row_operators_without_tokens(cb):
    lib = cb._lib
    assert lib.cobalt_permute_backward(None, None, 0, 2, 64, None, 0, None) == cb.OK
    assert lib.cobalt_layer_norm(None, None, None, 0, 64, 0, 1e-5, None, None, None, None) == cb.OK
    assert lib.cobalt_gate_topk(None, 0, 8, 2, 0, None, None, 0, None) == cb.OK
    assert lib.cobalt_gate_topk_backward(None, None, None, None, 0, 8, 2, 0, None, 0, None) == cb.OK
    assert lib.cobalt_dropout_add(None, None, 0, 0, 0.1, 1, None, 0, None) == cb.OK
    assert lib.cobalt_expert_ffn(None, None, None, 0, 2, 2, 64, 32, None, None, None, None, None, None, 0, None) == cb.OK
