"""Forms of linear's kernels that the size lists of the general tests do not reach: the epilogue of bf16 results without a residual or a
saved pre-activation, CTA pairs that compute several tiles, and a few tokens whose 8-bit rows do not fit in shared memory.

Bounds as in the general tests (u = 2^-24): a product's K terms are added in fp32, 2 K u sum|x w|; an activation's slope is at most
1.13, its own evaluation good to 2^-18 of its argument; then half a step of the result's type."""
import pytest
import torch

import dense_util as D

pytestmark = pytest.mark.gpu
U, BF16 = D.U, torch.bfloat16


def _rows8(t):
    """Rows in e4m3 with a scale each, as the plain form has them (pack_rows takes rows of up to 16384 values only)."""
    codes, scales = D.pack(t, torch.float8_e4m3fn, 0)
    return codes.float().to(torch.float8_e4m3fn), scales.float()


def _inputs(T, K, N, operand, seed):
    """x and w as the call takes them and their values; rows and features of different sizes, so that no bias or scale passes for
    another one."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def rnd(*s):
        return torch.randn(s, generator=g, device="cuda")

    x = (rnd(T, K) * torch.exp(0.5 * rnd(T, 1))).to(BF16)
    w = (rnd(N, K) * K ** -0.5 * torch.exp(0.5 * rnd(N, 1))).to(BF16)
    bias = (0.5 * rnd(N)).to(BF16)
    if operand == "e4m3":
        x, w = _rows8(x), _rows8(w)
        return x, w, D.values(*x, 0), D.values(*w, 0), bias
    return x, w, x.double(), w.double(), bias


def _workspace(T, K, N):
    import paper_2609_36959_b200 as cb
    return torch.full((cb.linear_workspace_bytes(T, K, N),), 0xAB, dtype=torch.uint8, device="cuda")


def _check(out, pre, size, act, residual=None):
    y = D.act(pre, act) + (0 if residual is None else residual.double())
    bound = 1.13 * size + 2.0 ** -18 * pre.abs() + 4 * U * y.abs()
    off = (out.double() - y).abs() - bound - D.HALF[out.dtype] * (y.abs() + bound)
    assert (off <= 0).all(), (float(off.max()), int((off > 0).sum()))


#           T     K     N
PLAIN = [(5, 48, 8), (31, 528, 136), (33, 80, 264), (70, 272, 72), (129, 1008, 200), (257, 272, 1032), (300, 4096, 264), (1000, 144, 40),
         (2100, 512, 776), (2400, 272, 6408), (5000, 80, 2824)]


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("operand", ["bf16", "e4m3"])
@pytest.mark.parametrize("T,K,N", PLAIN)
def test_plain_results_against_64_bits(T, K, N, operand, act):
    """bf16 results of bias and activation alone; the last two sizes give a pair several tiles, the last of them three or five chunks of 32
    tokens."""
    import paper_2609_36959_b200 as cb
    x, w, xd, wd, bias = _inputs(T, K, N, operand, T + K + N)
    ws, product = _workspace(T, K, N), xd @ wd.t()
    size = 2 * (K + 4) * U * (xd.abs() @ wd.abs().t()) + 1e-30
    for b in (bias, None):
        whole = torch.full((T + 1, N), 7.0, dtype=BF16, device="cuda")
        out = whole[:T]
        cb.linear(x, w, out, ws, bias=b, act=act)
        pre = product if b is None else product + b.double()
        _check(out, pre, size + 4 * U * pre.abs(), act)
        first = out.clone()
        for _ in range(3):
            out.fill_(5.0)
            cb.linear(x, w, out, ws, bias=b, act=act)
            assert torch.equal(out, first)
        assert (whole[T] == 7).all()
    assert cb.read_and_clear_device_error() == 0


@pytest.mark.parametrize("form", ["f32", "f32 residual", "residual", "pre bf16", "pre i8"])
@pytest.mark.parametrize("operand", ["bf16", "e4m3"])
@pytest.mark.parametrize("T,K,N", [(5000, 1072, 2824), (3001, 1104, 4104)])
def test_several_tiles_a_pair_against_64_bits(T, K, N, operand, form):
    """276 and 204 tiles on 74 pairs: accumulators, constants, token scales and staging are used again.  K is above 512, so that fp32
    results are added in several pieces a tile."""
    import paper_2609_36959_b200 as cb
    x, w, xd, wd, bias = _inputs(T, K, N, operand, T + K + N)
    dtype, ws, act = torch.float32 if form.startswith("f32") else BF16, _workspace(T, K, N), "silu" if form.startswith("pre") else "none"
    g = torch.Generator(device="cuda").manual_seed(8)
    residual = torch.randn((T, N), generator=g, device="cuda").to(dtype) if "residual" in form else None
    pre = None if act == "none" else torch.empty((T, N), dtype=BF16, device="cuda") if form == "pre bf16" else (
        torch.empty((T, N), dtype=torch.int8, device="cuda"), torch.empty((T, -(-N // 128)), device="cuda"))
    whole = torch.full((T + 1, N), 7.0, dtype=dtype, device="cuda")
    out = whole[:T]
    cb.linear(x, w, out, ws, bias=bias, residual=residual, act=act, pre=pre)
    ref = xd @ wd.t() + bias.double()
    size = 2 * (K + 4) * U * (xd.abs() @ wd.abs().t()) + 4 * U * ref.abs()
    _check(out, ref, size, act, residual)
    if isinstance(pre, tuple):
        step = D.values(torch.ones_like(ref), pre[1], 128)
        assert ((D.values(*pre, 128) - ref).abs() <= 0.5001 * step + size).all()
    elif pre is not None:
        assert ((pre.double() - ref).abs() <= D.HALF[BF16] * (ref.abs() + size) + size).all()
    first = out.clone()
    for _ in range(3):
        out.fill_(5.0)
        cb.linear(x, w, out, ws, bias=bias, residual=residual, act=act, pre=pre)
        assert torch.equal(out, first)
    assert (whole[T] == 7).all() and cb.read_and_clear_device_error() == 0


@pytest.mark.parametrize("T,K,N", [(300, 4104, 2824), (1000, 2824, 4104)])
def test_several_weight_gradient_tiles_a_pair(T, K, N):
    import paper_2609_36959_b200 as cb
    g = torch.Generator(device="cuda").manual_seed(T)
    x, dy = (torch.randn((T, c), generator=g, device="cuda").to(BF16) for c in (K, N))
    ref = dy.double().t() @ x.double()
    size = 2 * (T + 4) * U * (dy.double().abs().t() @ x.double().abs())
    whole, ws = torch.full((N + 1, K), 7.0, dtype=BF16, device="cuda"), _workspace(T, K, N)
    for _ in range(4):
        whole[:N] = 5.0
        cb.linear_backward(dy, x, None, ws, grad_w=whole[:N])
        assert ((whole[:N].double() - ref).abs() <= size + D.HALF[BF16] * (ref.abs() + size)).all()
    assert (whole[N] == 7).all() and cb.read_and_clear_device_error() == 0


@pytest.mark.parametrize("T,K,N", [(1, 28160, 264), (1, 28176, 264), (1, 65536, 24), (2, 14080, 136), (2, 14096, 136), (2, 40000, 72), (3, 9344, 264),
                                   (3, 9360, 264), (4, 9360, 264), (4, 65536, 40)])
def test_few_tokens_of_long_8_bit_rows(T, K, N):
    """On both sides of the widths at which the tokens, decoded to two bytes a value, no longer fit in a CTA's share of shared memory
    (55 KB for one token or two, 73 KB for four)."""
    import paper_2609_36959_b200 as cb
    x, w, xd, wd, bias = _inputs(T, K, N, "e4m3", T + K + N)
    ref = xd @ wd.t() + bias.double()
    size = 2 * (K + 4) * U * (xd.abs() @ wd.abs().t()) + 4 * U * ref.abs()
    g = torch.Generator(device="cuda").manual_seed(9)
    for dtype in (BF16, torch.float32):
        residual = torch.randn((T, N), generator=g, device="cuda").to(dtype)
        whole = torch.full((T + 1, N), 7.0, dtype=dtype, device="cuda")
        cb.linear(x, w, whole[:T], _workspace(T, K, N), bias=bias, residual=residual, act="relu")
        _check(whole[:T], ref, size, "relu", residual)
        assert (whole[T] == 7).all()
