"""The dense operators without a GPU: published vectors of the generator, gradients of the plain forms against
central differences, and the argument checks of the C entries, which run before any device work."""
import pytest
import torch

import layer_util as L


def test_philox_published_vectors():
    """Known answers of philox4x32-10 published with the generator (Salmon et al., SC 2011)."""
    ones = 0xFFFFFFFF
    assert L.philox_words((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert L.philox_words((ones,) * 4, (ones,) * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert L.philox_words((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0)) == [
        0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def _difference(f, at, direction, h=1e-5):
    return (f(at + h * direction) - f(at - h * direction)) / (2 * h)


def _close(a, b):
    # central differences in 64 bits with step 1e-5: truncation about 1e-10, cancellation about 1e-11 of |f|
    assert abs(float(a) - float(b)) <= 1e-6 * (1.0 + abs(float(b))), (float(a), float(b))


def test_plain_gradients_against_differences():
    g = torch.Generator().manual_seed(5)

    def rnd(*shape):
        return torch.randn(shape, generator=g, dtype=torch.float64)

    x, gamma, beta, dy = rnd(3, 24), rnd(24), rnd(24), rnd(3, 24)
    dx, dgamma, dbeta = L.norm_backward(dy, x, gamma, 1e-5)
    for at, grad, f in ((x, dx, lambda v: (L.norm_forward(v, gamma, beta, 1e-5)[0] * dy).sum()),
                        (gamma, dgamma, lambda v: (L.norm_forward(x, v, beta, 1e-5)[0] * dy).sum()),
                        (beta, dbeta, lambda v: (L.norm_forward(x, gamma, v, 1e-5)[0] * dy).sum())):
        v = rnd(*at.shape)
        _close((grad * v).sum(), _difference(f, at, v))
    logits, gw = 3 * rnd(4, 9), rnd(4, 3)
    for sigmoid in (False, True):
        ids, w, _ = L.gate_forward(logits, 3, sigmoid)
        v = rnd(4, 9)
        _close((L.gate_backward(gw, logits, ids, w, sigmoid) * v).sum(),
               _difference(lambda t: (L.gate_weights(t.gather(1, ids), sigmoid) * gw).sum(), logits, v))
    rows, wgu, wd, dy = rnd(7, 8), rnd(2, 12, 8), rnd(2, 8, 6), rnd(7, 8)
    ranges = [(0, 3, 1), (3, 4, 0), (4, 7, 1)]          # expert 1 sits in two slots: its gradients add up
    b = L.ffn_backward(dy, rows, ranges, wgu, wd)
    for at, grad, f in ((rows, b["dx"], lambda v: (L.ffn_forward(v, ranges, wgu, wd)[0] * dy).sum()),
                        (wgu, b["dgu"], lambda v: (L.ffn_forward(rows, ranges, v, wd)[0] * dy).sum()),
                        (wd, b["ddn"], lambda v: (L.ffn_forward(rows, ranges, wgu, v)[0] * dy).sum())):
        v = rnd(*at.shape)
        _close((grad * v).sum(), _difference(f, at, v))


@pytest.fixture(scope="module")
def cb():
    from paper_2609_36959_b200 import build
    build.build()
    import paper_2609_36959_b200.binding as binding
    return binding


def test_layer_norm_refusals(cb):
    lib, bad, un = cb._lib, cb.ERR_INVALID_ARG, cb.ERR_UNSUPPORTED

    def fwd(x=16, T=4, H=64, dtype=0, eps=1e-5, y=16):
        return lib.cobalt_layer_norm(x, 16, 16, T, H, dtype, eps, y, 16, 16, None)

    assert fwd(T=0) == cb.OK
    assert fwd(x=None) == fwd(y=None) == fwd(x=8) == fwd(T=-1) == fwd(H=0) == fwd(dtype=2) == bad
    assert fwd(eps=-1.0) == fwd(eps=float("nan")) == bad
    assert fwd(H=12) == fwd(H=16392) == fwd(T=1 << 31) == un
    assert cb.layer_norm_workspace_bytes(4, 12) == 0 and cb.layer_norm_workspace_bytes(1 << 20, 7168) % 256 == 0

    def bwd(dy=16, T=4, H=64, ws=16, nbytes=1 << 30, gg=16):
        return lib.cobalt_layer_norm_backward(dy, 16, 16, 16, 16, T, H, 0, 16, gg, 16, ws, nbytes, None)

    assert bwd(dy=None) == bwd(dy=4) == bwd(gg=None) == bwd(ws=8) == bad
    assert bwd(ws=None) == bwd(nbytes=16) == cb.ERR_WORKSPACE_TOO_SMALL
    assert bwd(H=20) == un


def test_gate_refusals(cb):
    lib, bad, un = cb._lib, cb.ERR_INVALID_ARG, cb.ERR_UNSUPPORTED

    def fwd(l=16, T=4, E=8, K=2, dtype=1, flags=0):
        return lib.cobalt_gate_topk(l, T, E, K, dtype, 16, 16, flags, None)

    assert fwd(T=0) == cb.OK
    assert fwd(l=None) == fwd(l=20) == fwd(K=0) == fwd(K=9) == fwd(E=0) == fwd(T=-1) == fwd(dtype=3) == fwd(flags=2) == bad
    assert fwd(E=1025) == fwd(E=32, K=17) == fwd(T=1 << 30) == un

    def bwd(g=16, l=16, flags=0, out=16):
        return lib.cobalt_gate_topk_backward(g, l, 16, 16, 4, 8, 2, 1, out, flags, None)

    assert bwd(g=None) == bwd(out=None) == bwd(l=None, flags=cb.GATE_SIGMOID) == bwd(g=24) == bwd(flags=4) == bad


def test_dropout_refusals(cb):
    lib, bad = cb._lib, cb.ERR_INVALID_ARG

    def fwd(x=16, n=8, dtype=0, p=0.5, seed=1, out=16, flags=0, r=None):
        return lib.cobalt_dropout_add(x, r, n, dtype, p, seed, out, flags, None)

    assert fwd(n=0) == cb.OK
    assert fwd(x=None) == fwd(out=None) == fwd(x=2) == fwd(r=6) == fwd(n=-1) == fwd(dtype=-1) == bad
    assert fwd(p=-0.1) == fwd(p=1.5) == fwd(p=float("nan")) == fwd(flags=1) == bad
    assert fwd(flags=cb.SEED_ON_DEVICE, seed=0) == fwd(flags=cb.SEED_ON_DEVICE, seed=12) == bad
    assert lib.cobalt_dropout_add_backward(None, 8, 0, 0.5, 1, 16, 0, None) == bad


def test_expert_ffn_refusals(cb):
    lib, bad, un, small = cb._lib, cb.ERR_INVALID_ARG, cb.ERR_UNSUPPORTED, cb.ERR_WORKSPACE_TOO_SMALL

    def fwd(rows=16, P=4, D=2, E=2, H=64, F=32, act=16, pre=None, out=16, ws=256, nbytes=1 << 30):
        return lib.cobalt_expert_ffn(rows, 16, 16, P, D, E, H, F, 16, 16, act, pre, out, ws, nbytes, None)

    assert fwd(P=0) == cb.OK
    assert fwd(rows=None) == fwd(act=None) == fwd(out=None) == fwd(rows=8) == fwd(pre=4) == fwd(ws=8) == bad
    assert fwd(P=-1) == fwd(D=0) == fwd(E=0) == fwd(H=0) == fwd(F=0) == bad
    assert fwd(H=12) == fwd(F=4) == fwd(D=5000) == fwd(E=1025) == fwd(P=1 << 31) == fwd(P=(1 << 31) - 1024) == fwd(H=65544) == un
    assert fwd(ws=None) == fwd(nbytes=0) == small
    assert cb.expert_ffn_workspace_bytes(4, 2, 2, 12, 32) == 0 and cb.expert_ffn_workspace_bytes(4, 2, 2, 64, 32) > 0

    def bwd(dy=16, gx=16, gu=16, gd=16, pre=16, ws=256, nbytes=1 << 30, P=4):
        return lib.cobalt_expert_ffn_backward(dy, 16, 16, 16, P, 2, 2, 64, 32, 16, 16, pre, 16, 16, gx, gu, gd, ws, nbytes, None)

    assert bwd(dy=None) == bwd(pre=None) == bwd(gx=None, gu=None, gd=None) == bwd(gx=8) == bad
    assert bwd(ws=None) == bwd(nbytes=8) == small


def test_binding_refuses_wrong_shapes_and_host_tensors(cb):
    z = torch.zeros
    with pytest.raises(TypeError):
        cb.layer_norm(z(2, 16), z(16), z(16), 1e-5, z(2, 16), z(2), z(2))
    with pytest.raises(cb.CobaltError):
        cb.layer_norm(z(2, 16), z(8), z(16), 1e-5, z(2, 16), z(2), z(2))
    with pytest.raises(TypeError):
        cb.gate_topk(z(2, 16, dtype=torch.float16), z(2, 2, dtype=torch.int32), z(2, 2))
    with pytest.raises(cb.CobaltError):
        cb.gate_topk(z(2, 16), z(3, 2, dtype=torch.int32), z(3, 2))
    with pytest.raises(cb.CobaltError):
        cb.dropout_add(z(4), z(5), 0.1, 1, z(4))
    with pytest.raises(cb.CobaltError):
        cb.expert_ffn(z(4, 16), z(3, dtype=torch.int32), z(2, dtype=torch.int32), z(2, 16, 16), z(2, 16, 16), z(4, 16), z(4, 16), z(256))
