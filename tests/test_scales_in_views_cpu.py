"""The boundaries of scales and rstd that the C entries take: any of 4 bytes where they are read or written one value at a time."""
import pytest


@pytest.fixture(scope="module")
def cb():
    from paper_2609_36959_b200 import build
    build.build()
    import paper_2609_36959_b200.binding as binding
    return binding


def test_scales_on_4_byte_boundaries(cb):
    """A workspace that is too small is found after the pointers' checks, and before any device work."""
    lib, bad, small = cb._lib, cb.ERR_INVALID_ARG, cb.ERR_WORKSPACE_TOO_SMALL

    def linear(xs, ws=16):
        return lib.cobalt_linear(16, xs, 16, ws, None, None, 4, 64, 32, cb.E4M3, 0, 0, None, None, 0, 16, 256, 0, None)

    assert linear(16) == linear(20) == linear(28) == small and linear(18) == linear(17) == linear(20, 20) == bad

    def norm_backward(scales, rstd):
        return lib.cobalt_rms_norm_backward(16, None, 16, scales, cb.I8, 128, 16, rstd, 4, 64, 0, 16, 16, 256, 0, None)

    assert norm_backward(20, 16) == norm_backward(16, 20) == norm_backward(28, 24) == small
    assert norm_backward(18, 16) == norm_backward(16, 18) == bad

    def norm(scales):
        return lib.cobalt_rms_norm(16, None, 16, 4, 64, 0, 1e-5, None, None, 16, scales, cb.I8, 128, None, None)

    assert norm(18) == norm(17) == bad
