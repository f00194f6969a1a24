"""The operators on token rows without a GPU: gradients of the plain forms against central differences, and the argument checks
of the C entries and of the binding, which run before any device work."""
import pytest
import torch

import dense_util as D


@pytest.fixture(scope="module")
def cb():
    from paper_2609_36959_b200 import build
    build.build()
    import paper_2609_36959_b200.binding as binding
    return binding


def test_plain_gradients_against_differences():
    g = torch.Generator().manual_seed(5)

    def rnd(*shape):
        return torch.randn(shape, generator=g, dtype=torch.float64)

    def close(grad, at, f):
        v, h = rnd(*at.shape), 1e-5
        a, b = float((grad * v).sum()), float((f(at + h * v) - f(at - h * v)) / (2 * h))
        assert abs(a - b) <= 1e-6 * (1 + abs(b)), (a, b)      # truncation about 1e-10, cancellation about 1e-11 of |f|

    s, gamma, dy, ds = rnd(3, 24), rnd(24), rnd(3, 24), rnd(3, 24)
    rstd = D.rms_forward(s, gamma, 1e-5)[1]
    dx, dgamma = D.rms_backward(dy, s, gamma, rstd, ds)
    close(dx, s, lambda v: (D.rms_forward(v, gamma, 1e-5)[0] * dy + v * ds).sum())
    close(dgamma, gamma, lambda v: (D.rms_forward(s, v, 1e-5)[0] * dy).sum())
    v = torch.cat([rnd(40), torch.tensor([0.7, -0.7], dtype=torch.float64)])
    for kind in ("none", "relu", "silu", "gelu"):
        close(D.act_slope(v, kind), v, lambda t: D.act(t, kind).sum())
    x, w, dy = rnd(5, 16), rnd(24, 16), rnd(5, 24)
    d = dy * D.act_slope(x @ w.t(), "gelu")
    close(d @ w, x, lambda t: (D.act(t @ w.t(), "gelu") * dy).sum())
    close(d.t() @ x, w, lambda t: (D.act(x @ t.t(), "gelu") * dy).sum())


def test_codes_of_the_definition():
    """The table of e4m3's values: every code is its own nearest one, halves go to the even neighbour, and int8 by rounding."""
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    every = every[torch.isfinite(every)]
    assert torch.equal(D.nearest_code(every, torch.float8_e4m3fn), every)
    up = torch.sort(every[every >= 0].unique()).values
    middle = (up[1:] + up[:-1]) / 2
    got = D.nearest_code(middle, torch.float8_e4m3fn)
    even = torch.where(torch.arange(len(middle)) % 2 == 0, up[:-1], up[1:])
    assert torch.equal(got, even)
    assert D.nearest_code(torch.tensor([0.5, 1.5, -2.5, 126.5]), torch.int8).tolist() == [0, 2, -2, 126]


def test_pack_refusals(cb):
    lib, bad, un = cb._lib, cb.ERR_INVALID_ARG, cb.ERR_UNSUPPORTED

    def pack(x=16, T=4, H=64, dtype=0, code=2, group=128, q=16, s=16):
        return lib.cobalt_pack_rows(x, T, H, dtype, code, group, q, s, None)

    def unpack(q=16, s=16, T=4, H=64, code=2, group=128, dtype=0, out=16):
        return lib.cobalt_unpack_rows(q, s, T, H, code, group, dtype, out, None)

    for call in (pack, unpack):
        assert call(T=0) == cb.OK
        assert call(T=-1) == call(H=0) == call(dtype=2) == call(code=1) == call(code=4) == call(group=64) == bad
        assert call(q=None) == call(s=None) == call(q=8) == call(s=4) == bad
        assert call(H=12) == call(H=16392) == call(T=1 << 31) == un
    assert pack(x=None) == pack(x=8) == unpack(out=None) == unpack(out=8) == bad


def test_rms_norm_refusals(cb):
    lib, bad, un, small = cb._lib, cb.ERR_INVALID_ARG, cb.ERR_UNSUPPORTED, cb.ERR_WORKSPACE_TOO_SMALL

    def fwd(x=16, r=None, T=4, H=64, dtype=0, eps=1e-5, total=None, y=16, q=None, s=None, code=0, group=0, rstd=None):
        return lib.cobalt_rms_norm(x, r, 16, T, H, dtype, eps, total, y, q, s, code, group, rstd, None)

    assert fwd(T=0) == cb.OK
    assert fwd(x=None) == fwd(y=None) == fwd(x=8) == fwd(rstd=4) == fwd(T=-1) == fwd(H=0) == fwd(dtype=2) == bad
    assert fwd(eps=-1.0) == fwd(eps=float("nan")) == fwd(total=16) == fwd(r=16, total=32, y=32) == bad
    assert fwd(q=16) == fwd(q=16, s=16, code=1) == fwd(q=16, s=16, code=2, group=32) == fwd(q=16, code=2, group=128) == bad
    assert fwd(H=12) == fwd(H=16392) == fwd(T=1 << 31) == un

    def bwd(dy=16, rows=16, scales=None, kind=0, group=0, T=4, H=64, ws=256, nbytes=1 << 30, gg=16, ds=None):
        return lib.cobalt_rms_norm_backward(dy, ds, rows, scales, kind, group, 16, 16, T, H, 0, 16, gg, ws, nbytes, None)

    assert bwd(dy=None) == bwd(rows=None) == bwd(gg=None) == bwd(ds=4) == bwd(ws=8) == bad
    assert bwd(kind=1) == bwd(kind=3, group=5, scales=16) == bwd(kind=3, group=128) == bwd(kind=4, scales=16) == bad
    assert bwd(ws=None) == bwd(nbytes=16) == small
    assert bwd(H=20) == un
    assert cb.rms_norm_workspace_bytes(4, 12) == 0 and cb.rms_norm_workspace_bytes(1 << 20, 7168) % 256 == 0


def test_linear_refusals(cb):
    lib, bad, un, small = cb._lib, cb.ERR_INVALID_ARG, cb.ERR_UNSUPPORTED, cb.ERR_WORKSPACE_TOO_SMALL

    def fwd(x=16, xs=None, w=16, ws_=None, bias=None, r=None, T=4, K=64, N=32, op=0, act=0, out_type=0, pre=None, ps=None, kind=0, out=16,
            ws=256, nbytes=1 << 40):
        return lib.cobalt_linear(x, xs, w, ws_, bias, r, T, K, N, op, act, out_type, pre, ps, kind, out, ws, nbytes, None)

    assert fwd(T=0) == cb.OK
    assert fwd(x=None) == fwd(w=None) == fwd(out=None) == fwd(x=8) == fwd(bias=2) == fwd(r=4) == fwd(ws=8) == bad
    assert fwd(op=1) == fwd(op=3) == fwd(op=2) == fwd(op=2, xs=16) == fwd(act=4) == fwd(act=-1) == fwd(out_type=2) == bad
    assert fwd(pre=16, kind=1) == fwd(pre=16, kind=3) == fwd(pre=8) == fwd(T=-1) == fwd(K=0) == fwd(N=0) == bad
    assert fwd(K=12) == fwd(N=12) == fwd(K=65544) == fwd(N=65544) == fwd(T=1 << 31) == fwd(op=2, xs=16, ws_=16, K=24) == un
    assert fwd(ws=None) == fwd(nbytes=0) == small

    def bwd(dy=16, x=16, w=16, pre=None, ps=None, kind=0, T=4, K=64, N=32, act=0, gt=0, gp=None, gx=16, gw=16, gb=16, ws=256, nbytes=1 << 40):
        return lib.cobalt_linear_backward(dy, x, w, pre, ps, kind, T, K, N, act, gt, gp, gx, gw, gb, ws, nbytes, None)

    assert bwd(dy=None) == bwd(x=None) == bwd(w=None) == bwd(gx=None, gw=None, gb=None) == bwd(gx=8) == bwd(gt=2) == bwd(act=9) == bad
    assert bwd(act=1, pre=None, gp=16) == bwd(act=1, pre=16) == bwd(act=1, pre=16, gp=16, kind=1) == bwd(act=1, pre=16, gp=16, kind=3) == bad
    assert bwd(gt=1) == bad                                   # fp32 gradients need their bf16 copy
    assert bwd(ws=None) == bwd(nbytes=0) == small
    assert bwd(K=20) == un
    assert cb.linear_workspace_bytes(4, 12, 8) == 0 and cb.linear_workspace_bytes(4096, 4096, 4096) % 256 == 0


def test_workspace_covers_the_plan_everywhere(cb):
    """The split products' parts and the bias's partial sums never need more than the query says: both bounds are arithmetic, so
    that a call is refused for its workspace exactly below the query's size."""
    for T, K, N in ((1, 8, 8), (5, 65536, 8), (4096, 64, 64), (131072, 7168, 256), (300, 16384, 16384), (1 << 20, 8, 16)):
        size = cb.linear_workspace_bytes(T, K, N)
        call = cb._lib.cobalt_linear(16, None, 16, None, None, None, T, K, N, 0, 0, 0, None, None, 0, 16, 256, size - 1, None)
        assert call == cb.ERR_WORKSPACE_TOO_SMALL and size >= 256


def test_a_workspace_for_many_tokens_serves_fewer(cb):
    sizes = [1, 2, 5, 64, 300, 801, 4099, 9473, 75776, 131072, 1 << 20]
    for K, N in ((8, 8), (4096, 2816), (7168, 256), (65536, 65536), (200, 1000), (40000, 8)):
        for query in (lambda t: cb.linear_workspace_bytes(t, K, N), lambda t: cb.rms_norm_workspace_bytes(t, min(K, 16384))):
            got = [query(t) for t in sizes + list(range(1, 4000, 17))]
            by_size = [b for _, b in sorted(zip(sizes + list(range(1, 4000, 17)), got))]
            assert by_size == sorted(by_size)


def test_binding_refuses_wrong_shapes_and_host_tensors(cb):
    z, f8 = torch.zeros, torch.float8_e4m3fn
    with pytest.raises(TypeError):
        cb.rms_norm(z(2, 16), z(16), 1e-5, y=z(2, 16))
    with pytest.raises(TypeError):
        cb.pack_rows(z(2, 16), z(2, 16, dtype=torch.uint8), z(2, 1))
    with pytest.raises(cb.CobaltError):
        cb.pack_rows(z(2, 512), z(2, 512, dtype=torch.int8), z(2, 3))
    with pytest.raises(cb.CobaltError):
        cb.unpack_rows(z(2, 512, dtype=torch.int8), z(3, 4), z(2, 512))
    with pytest.raises(TypeError):
        cb.linear(z(2, 16), (z(8, 16, dtype=f8), z(8, 1)), z(2, 8), z(256))
    with pytest.raises(TypeError):
        cb.linear(z(2, 16, dtype=torch.bfloat16), z(8, 16, dtype=torch.bfloat16), z(2, 8), z(256))
    with pytest.raises(ValueError):
        cb._activation("tanh")
