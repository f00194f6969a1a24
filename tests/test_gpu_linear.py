"""linear and its gradients against the 64-bit plain form.

Bounds (u = 2^-24): a product's K terms are added in fp32, each addition off by at most 2 u of what has been added (the tensor
cores may cut instead of rounding): 2 K u sum|x w|.  An activation's slope is at most 1.13; its own evaluation is good to 2^-18
of its argument.  Results add half a step of their type, the saved pre-activation likewise.  The gradients' products are checked
on d as the call left it in grad_pre (exact operands), and d on the saved pre-activation as it was left."""
import pytest
import torch

import dense_util as D

pytestmark = pytest.mark.gpu
U = D.U
BF16 = torch.bfloat16
#          T     K     N
SIZES = [(1, 8, 8), (1, 1032, 520), (2, 64, 128), (4, 2048, 72), (7, 200, 24), (31, 520, 136), (33, 72, 256), (129, 1000, 200), (257, 264, 1032), (300, 4096, 264),
         (1000, 136, 40), (2100, 512, 776)]


def _rows8(t):
    import paper_2609_36959_b200 as cb
    q, scales = torch.empty(t.shape, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty((t.shape[0], 1), device="cuda")
    cb.pack_rows(t, q, scales)
    return q, scales


def _inputs(T, K, N, seed, out=BF16):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def rnd(*s):
        return torch.randn(s, generator=g, device="cuda")

    return rnd(T, K).to(BF16), (rnd(N, K) * K ** -0.5).to(BF16), (0.3 * rnd(N)).to(BF16), rnd(T, N).to(out), rnd(T, N).to(out)


def _workspace(T, K, N):
    import paper_2609_36959_b200 as cb
    return torch.full((cb.linear_workspace_bytes(T, K, N),), 0xAB, dtype=torch.uint8, device="cuda")


def _guarded(T, N, dtype):
    """T rows of a buffer with one row behind them."""
    t = torch.full((T + 1, N), 7.0, dtype=dtype, device="cuda")
    return t, t[:T]


def _check_pre(pre, ref, tol):
    """The saved pre-activation's values (64 bits), within its format's half step of the product."""
    if isinstance(pre, tuple):
        got, step = D.values(pre[0], pre[1], 128), D.values(torch.ones_like(ref), pre[1], 128)
        assert ((got - ref).abs() <= 0.5001 * step + tol).all()
    else:
        got = pre.double()
        assert ((got - ref).abs() <= D.HALF[BF16] * (ref.abs() + tol) + tol).all()
    return got


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("operand", ["bf16", "e4m3"])
@pytest.mark.parametrize("T,K,N", SIZES)
def test_linear_against_plain(T, K, N, operand, act):
    import paper_2609_36959_b200 as cb
    K = -(-K // 16) * 16 if operand == "e4m3" else K
    ws = _workspace(T, K, N)
    for out_type, use_bias, use_residual, pre_type in ((BF16, True, True, None), (BF16, True, False, "bf16"), (torch.float32, False, True, "i8")):
        x, w, bias, residual, _ = _inputs(T, K, N, T * 31 + K + N, out_type)
        bias, residual = bias if use_bias else None, residual if use_residual else None
        xd, wd = x.double(), w.double()
        if operand == "e4m3":
            x, w = _rows8(x), _rows8(w)
            xd, wd = D.values(*x, 0), D.values(*w, 0)
        pre = None if pre_type is None else torch.empty((T, N), dtype=BF16, device="cuda") if pre_type == "bf16" else (
            torch.empty((T, N), dtype=torch.int8, device="cuda"), torch.empty((T, -(-N // 128)), device="cuda"))
        whole, out = _guarded(T, N, out_type)
        cb.linear(x, w, out, ws, bias=bias, residual=residual, act=act, pre=pre)
        torch.cuda.synchronize()
        assert (whole[T] == 7).all() and cb.read_and_clear_device_error() == 0
        ref = xd @ wd.t() + (0 if bias is None else bias.double())
        tol = 2 * (K + 4) * U * (xd.abs() @ wd.abs().t()) + 4 * U * ref.abs() + 1e-30
        if pre is not None:
            _check_pre(pre, ref, tol)
        y = D.act(ref, act) + (0 if residual is None else residual.double())
        bound = 1.13 * tol + 2.0 ** -18 * ref.abs() + 4 * U * y.abs()
        assert ((out.double() - y).abs() <= bound + D.HALF[out_type] * (y.abs() + bound)).all(), (out_type, float((out.double() - y).abs().max()))
        again = torch.empty_like(out)
        cb.linear(x, w, again, ws, bias=bias, residual=residual, act=act, pre=pre)
        assert torch.equal(again, out)                                    # the same bits every time


def test_linear_sums_in_32_bits():
    """The roundings of a long sum are independent: far below their sum. 448 groups of sixteen terms, each rounded or cut by at
    most 2 u of a running sum no larger than about three times the result's rms: 2 u * 3 * sqrt(448) = 7.6e-6."""
    import paper_2609_36959_b200 as cb
    for T, N in ((3, 264), (520, 256), (5000, 256)):
        x, w, _, _, _ = _inputs(T, 7168, N, 5, torch.float32)
        out = torch.empty((T, N), device="cuda")
        cb.linear(x, w, out, _workspace(T, 7168, N))
        ref = x.double() @ w.double().t()
        assert float((out.double() - ref).norm() / ref.norm()) < 7.6e-6


@pytest.mark.parametrize("act,pre_type", [("none", None), ("relu", "bf16"), ("silu", "i8"), ("silu", "bf16"), ("gelu", "i8"), ("gelu", "bf16")])
@pytest.mark.parametrize("T,K,N", SIZES)
def test_linear_gradients_against_plain(T, K, N, act, pre_type):
    import paper_2609_36959_b200 as cb
    ws = _workspace(T, K, N)
    for grad_type in (BF16, torch.float32):
        x, w, bias, _, dy = _inputs(T, K, N, T * 17 + K + N, grad_type)
        pre = None if pre_type is None else torch.empty((T, N), dtype=BF16, device="cuda") if pre_type == "bf16" else (
            torch.empty((T, N), dtype=torch.int8, device="cuda"), torch.empty((T, -(-N // 128)), device="cuda"))
        cb.linear(x, w, torch.empty((T, N), dtype=BF16, device="cuda"), ws, bias=bias, act=act, pre=pre)
        (wx, gx), (ww, gw), (wp, gp) = _guarded(T, K, BF16), _guarded(N, K, BF16), _guarded(T, N, BF16)
        gb = torch.full((N,), 7.0, dtype=BF16, device="cuda")
        cb.linear_backward(dy, x, w, ws, act=act, pre=pre, grad_pre=gp, grad_x=gx, grad_w=gw, grad_bias=gb)
        torch.cuda.synchronize()
        assert (wx[T] == 7).all() and (ww[N] == 7).all() and (wp[T] == 7).all() and cb.read_and_clear_device_error() == 0
        # d on the saved pre-activation
        saved = None if pre is None else D.values(*pre, 128) if isinstance(pre, tuple) else pre.double()
        d = dy.double() * (1.0 if act == "none" else D.act_slope(saved, act))
        off = 0 if act == "none" else 2.0 ** -18 * dy.double().abs() * (1 + saved.abs())
        if act == "none" and grad_type == BF16:
            used = dy.double()
        else:
            used = gp.double()
            assert ((used - d).abs() <= D.HALF[BF16] * (d.abs() + off) + off).all()
        ref = d.sum(0)
        tol = (T + 64) * U * d.abs().sum(0) + (0 if act == "none" else off.sum(0))
        assert ((gb.double() - ref).abs() <= D.HALF[BF16] * (ref.abs() + tol) + tol).all()
        # the products, of exact operands
        for got, ref, size in ((gx, used @ w.double(), 2 * (N + 4) * U * (used.abs() @ w.double().abs())),
                               (gw, used.t() @ x.double(), 2 * (T + 4) * U * (used.abs().t() @ x.double().abs()))):
            assert ((got.double() - ref).abs() <= size + D.HALF[BF16] * (ref.abs() + size) + 1e-30).all()
        # each result by itself, d over the bf16 gradient
        if grad_type == BF16:
            for name, like in (("grad_x", gx), ("grad_w", gw), ("grad_bias", gb)):
                one, over = torch.empty_like(like), dy.clone()
                cb.linear_backward(over, x if name == "grad_w" else None, w if name == "grad_x" else None, ws, act=act, pre=pre, grad_pre=over, **{name: one})
                assert torch.equal(one, like)


@pytest.mark.parametrize("T,K,N", [(75777, 1032, 136), (80000, 2056, 256), (75800, 1024, 8)])
def test_linear_gradient_of_many_rows_from_a_few_features(T, K, N):
    """A router's dx: few blocks of the summed extent, many tokens; rows at the ends and in between checked one by one."""
    import paper_2609_36959_b200 as cb
    _, w, _, _, dy = _inputs(T, K, N, 3)
    whole, gx = _guarded(T, K, BF16)
    for _ in range(2):
        gx.fill_(5.0)
        cb.linear_backward(dy, None, w, _workspace(T, K, N), grad_x=gx)
    torch.cuda.synchronize()
    assert (whole[T] == 7).all() and cb.read_and_clear_device_error() == 0
    for part in (slice(0, 20000), slice(30000, 50000), slice(T - 26000, T)):
        ref = dy[part].double() @ w.double()
        size = 2 * (N + 4) * U * (dy[part].double().abs() @ w.double().abs())
        assert ((gx[part].double() - ref).abs() <= size + D.HALF[BF16] * (ref.abs() + size)).all()


@pytest.mark.parametrize("T,K,N", [(1457, 8192, 264), (449, 16384, 520), (2400, 6400, 136)])
def test_linear_tiles_with_an_odd_number_of_chunks(T, K, N):
    """Last tiles of 177, 193 and 96 rows: a group of warps stores an odd number of chunks, and the pair's next tile follows at once."""
    import paper_2609_36959_b200 as cb
    _, w, _, _, dy = _inputs(T, K, N, 3)
    ref = dy.double() @ w.double()
    size = 2 * (N + 4) * U * (dy.double().abs() @ w.double().abs()) + D.HALF[BF16] * ref.abs() * 1.001
    gx, ws = torch.empty((T, K), dtype=BF16, device="cuda"), _workspace(T, K, N)
    for _ in range(10):
        gx.fill_(5.0)
        cb.linear_backward(dy, None, w, ws, grad_x=gx)
        assert ((gx.double() - ref).abs() <= size).all()


def test_linear_rows_keep_to_themselves():
    """A row of x with a NaN or an infinity reaches its own row of the result only; one of W its own column."""
    import paper_2609_36959_b200 as cb
    for T in (3, 70, 300):
        x, w, _, _, _ = _inputs(T, 264, 136, T)
        x[1, 5], w[7, 3] = float("nan"), float("inf")
        out = torch.empty((T, 136), dtype=BF16, device="cuda")
        cb.linear(x, w, out, _workspace(T, 264, 136))
        bad = ~torch.isfinite(out)
        want = torch.zeros_like(bad)
        want[1], want[:, 7] = True, True
        assert torch.equal(bad, want)


def test_linear_in_place_residual_and_no_rows():
    import paper_2609_36959_b200 as cb
    x, w, bias, residual, _ = _inputs(70, 264, 136, 3)
    out, ws = torch.empty_like(residual), _workspace(70, 264, 136)
    cb.linear(x, w, out, ws, bias=bias, residual=residual, act="gelu")
    cb.linear(x, w, residual, ws, bias=bias, residual=residual, act="gelu")
    assert torch.equal(out, residual)
    gw, gb = torch.full((136, 264), 7.0, dtype=BF16, device="cuda"), torch.full((136,), 7.0, dtype=BF16, device="cuda")
    cb.linear(x[:0], w, out[:0], ws)
    cb.linear_backward(out[:0], x[:0], w, ws, grad_w=gw, grad_bias=gb)
    torch.cuda.synchronize()
    assert (gw == 0).all() and (gb == 0).all()


def test_linear_captured_with_two_streams():
    """Captured calls replay on changed inputs; two captured calls with a workspace each may run side by side."""
    import paper_2609_36959_b200 as cb
    sets = []
    for i in range(2):
        x, w, bias, residual, dy = _inputs(200, 520, 264, 10 + i)
        b = {"out": torch.empty_like(dy), "ws": _workspace(200, 520, 264), "pre": (torch.empty((200, 264), dtype=torch.int8, device="cuda"),
                                                                                    torch.empty((200, 3), device="cuda")),
             "gp": torch.empty_like(dy), "gx": torch.empty_like(x), "gw": torch.empty_like(w), "gb": torch.empty_like(bias)}
        sets.append((x, w, bias, residual, dy, b))

    def step(x, w, bias, residual, dy, b):
        cb.linear(x, w, b["out"], b["ws"], bias=bias, residual=residual, act="silu", pre=b["pre"])
        cb.linear_backward(dy, x, w, b["ws"], act="silu", pre=b["pre"], grad_pre=b["gp"], grad_x=b["gx"], grad_w=b["gw"], grad_bias=b["gb"])

    for s in sets:
        step(*s)
    graphs, streams = [], [torch.cuda.Stream() for _ in sets]
    for s, stream in zip(sets, streams):
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step(*s)
        graphs.append(graph)
    for s in sets:
        s[0].neg_()
    torch.cuda.synchronize()
    for graph, stream in zip(graphs, streams):
        with torch.cuda.stream(stream):
            graph.replay()
    torch.cuda.synchronize()
    for x, w, bias, residual, dy, b in sets:
        got = [b[k].clone() for k in ("out", "gx", "gw", "gb")]
        step(x, w, bias, residual, dy, b)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b[k]) for a, k in zip(got, ("out", "gx", "gw", "gb")))


def test_linear_smallest_pre_activations_in_8_bits():
    """Pre-activations so small that 127 / most is past the range, zeros among them: the bias alone, as x is 0, so that pre is exact.  The
    scale, below 2^-126, is good to 2^-150."""
    import paper_2609_36959_b200 as cb
    T, K, N = 40, 64, 264
    g = torch.Generator(device="cuda").manual_seed(1)
    bias = (torch.randint(-9, 10, (N,), generator=g, device="cuda").double() * 2.0 ** -129).to(BF16)
    pre = torch.full((T, N), 7, dtype=torch.int8, device="cuda"), torch.full((T, 3), 7.0, device="cuda")
    out = torch.empty((T, N), dtype=BF16, device="cuda")
    cb.linear(torch.zeros((T, K), dtype=BF16, device="cuda"), torch.ones((N, K), dtype=BF16, device="cuda"), out, _workspace(T, K, N), bias=bias,
              act="silu", pre=pre)
    ref = bias.double().expand(T, N)
    step = D.values(torch.ones_like(ref), pre[1], 128)
    assert ((D.values(pre[0], pre[1], 128) - ref).abs() <= 0.5 * step * (1 + 64 * U) + 127 * 2.0 ** -150).all()


def test_linear_bias_gradient_alone_takes_the_workspace_of_the_whole_call():
    """Neither x nor w is given then, so that the call does not know the rows' width; and a workspace for many tokens serves fewer."""
    import paper_2609_36959_b200 as cb
    T, K, N = 8192, 4096, 2816
    ws = _workspace(T, K, N)
    for t in (T, 801, 300, 1):
        dy = torch.randn((t, N), generator=torch.Generator(device="cuda").manual_seed(t), device="cuda").to(BF16)
        got = torch.empty(N, dtype=BF16, device="cuda")
        cb.linear_backward(dy, None, None, ws, grad_bias=got)
        ref = dy.double().sum(0)
        assert ((got.double() - ref).abs() <= t * U * dy.double().abs().sum(0) + D.HALF[BF16] * ref.abs() * 1.001).all()


@pytest.mark.parametrize("K,N", [(16384, 264), (14080, 24), (13056, 520), (16, 8), (4096, 5000)])
def test_linear_one_token_from_8_bit_rows(K, N):
    """Widths on both sides of what fits in shared memory, and features that no CTA number divides.  bf16 results: half a step."""
    import paper_2609_36959_b200 as cb
    x, w, bias, residual, _ = _inputs(1, K, N, K + N)
    x8, w8 = _rows8(x), _rows8(w)
    out = torch.full((2, N), 7.0, dtype=BF16, device="cuda")
    cb.linear(x8, w8, out[:1], _workspace(1, K, N), bias=bias, residual=residual)
    xv, wv = D.values(*x8, 0), D.values(*w8, 0)
    ref = xv @ wv.t() + bias.double() + residual.double()
    tol = 2 * (K + 4) * U * (xv.abs() @ wv.abs().t() + bias.double().abs() + residual.double().abs()) + D.HALF[BF16] * ref.abs() * 1.001
    assert ((out[:1].double() - ref).abs() <= tol).all() and (out[1] == 7).all()
