"""Element offsets beyond 2^31 and 2^32: the far end of a large call equals a small call on the same values, bit for bit."""
import pytest
import torch

import layer_util as L

pytestmark = pytest.mark.gpu


def _same(a, b):
    assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def test_dropout_beyond_two_to_the_32():
    import paper_2609_36959_b200 as cb
    n, p, seed = (1 << 32) + 61, 0.5, 77
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    cb.dropout_add(x, None, p, seed, x)
    first = (n - 4001) // 8
    keep, scale = L.dropout_keep(n - 8 * first, p, seed, first_block=first)
    assert (x[8 * first:].float().cpu() == torch.tensor(keep, dtype=torch.float32) * scale).all()


def test_norm_beyond_two_to_the_32():
    import paper_2609_36959_b200 as cb
    T, H, tail = (1 << 32) // 4096 + 37, 4096, 8000      # enough rows for the same kernels in both calls
    dev = "cuda"
    x = torch.zeros((T, H), dtype=torch.bfloat16, device=dev)
    x[-tail:] = torch.randn((tail, H), device=dev).to(torch.bfloat16)
    gamma, beta = torch.rand(H, device=dev), torch.rand(H, device=dev)

    def run(xx):
        n = xx.shape[0]
        y, mean, rstd = torch.empty_like(xx), torch.empty(n, device=dev), torch.empty(n, device=dev)
        cb.layer_norm(xx, gamma, beta, 1e-5, y, mean, rstd)
        dx, dg, db = torch.empty_like(xx), torch.empty(H, device=dev), torch.empty(H, device=dev)
        ws = torch.empty(cb.layer_norm_workspace_bytes(n, H), dtype=torch.uint8, device=dev)
        cb.layer_norm_backward(xx, xx, gamma, mean, rstd, dx, dg, db, ws)
        return y, dx

    small_y, small_dx = run(x[-tail:].clone())
    y, dx = run(x)
    torch.cuda.synchronize()
    _same(y[-tail:], small_y)
    _same(dx[-tail:], small_dx)


def test_gate_beyond_two_to_the_31():
    import paper_2609_36959_b200 as cb
    T, E, K, tail = (1 << 31) // 1024 + 33, 1024, 4, 100
    logits = torch.zeros((T, E), dtype=torch.bfloat16, device="cuda")
    logits[-tail:] = torch.randn((tail, E), device="cuda").to(torch.bfloat16)
    g = torch.randn((T, K), device="cuda")

    def run(l, gg):
        ids, w = torch.empty((l.shape[0], K), dtype=torch.int32, device="cuda"), torch.empty((l.shape[0], K), device="cuda")
        grad = torch.empty_like(l)
        cb.gate_topk(l, ids, w, flags=cb.GATE_SIGMOID)
        cb.gate_topk_backward(gg, l, ids, w, grad, flags=cb.GATE_SIGMOID)
        return ids, w, grad

    small = run(logits[-tail:].clone(), g[-tail:].clone())
    for a, b in zip(run(logits, g), small):
        _same(a[-tail:], b)


def _ffn(rows, offsets, slots, wgu, wd, dy):
    import paper_2609_36959_b200 as cb
    (P, H), (E, _, F) = rows.shape, wd.shape

    def new(*s):
        return torch.empty(s, dtype=torch.bfloat16, device="cuda")

    act, out, pre, dpre, dx, dgu, ddn = new(P, F), new(P, H), new(P, 2 * F), new(P, 2 * F), new(P, H), new(E, 2 * F, H), new(E, H, F)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    slot = torch.tensor(slots, dtype=torch.int32, device="cuda")
    ws = torch.empty(cb.expert_ffn_workspace_bytes(P, len(slots), E, H, F), dtype=torch.uint8, device="cuda")
    cb.expert_ffn(rows, off, slot, wgu, wd, act, out, ws, pre=pre)
    cb.expert_ffn_backward(dy, rows, off, slot, wgu, wd, pre, act, dpre, ws, grad_rows=dx, grad_w_gate_up=dgu, grad_w_down=ddn)
    torch.cuda.synchronize()
    assert cb.read_and_clear_device_error() == 0
    return out, dx, dgu, ddn


def test_expert_ffn_rows_beyond_two_to_the_31():
    P, H, F, tail = (1 << 31) // 1024 + 300, 1024, 16, 77
    rows = torch.zeros((P, H), dtype=torch.bfloat16, device="cuda")
    dy = torch.zeros((P, H), dtype=torch.bfloat16, device="cuda")
    rows[-tail:], dy[-tail:] = torch.randn((tail, H), device="cuda").to(torch.bfloat16), torch.randn((tail, H), device="cuda").to(torch.bfloat16)
    wgu, wd = (torch.randn(s, device="cuda").to(torch.bfloat16) * 0.1 for s in ((2, 2 * F, H), (2, H, F)))
    small = _ffn(rows[-tail:].clone(), [0, 0, tail], [0, 1], wgu, wd, dy[-tail:].clone())
    large = _ffn(rows, [0, P - tail, P], [0, 1], wgu, wd, dy)
    for a, b in zip(large[:2], small[:2]):
        _same(a[-tail:], b)
    for a, b in zip(large[2:], small[2:]):
        _same(a[1], b[1])


@pytest.mark.parametrize("n", [5, 90])
def test_expert_ffn_weights_beyond_two_to_the_31(n):
    E, H, F = 300, 8192, 512
    wgu = torch.zeros((E, 2 * F, H), dtype=torch.bfloat16, device="cuda")
    wd = torch.zeros((E, H, F), dtype=torch.bfloat16, device="cuda")
    wgu[-1], wd[-1] = torch.randn((2 * F, H), device="cuda") * H ** -0.5, torch.randn((H, F), device="cuda") * F ** -0.5
    rows, dy = (torch.randn((n, H), device="cuda").to(torch.bfloat16) for _ in range(2))
    small = _ffn(rows, [0, n], [0], wgu[-1:].clone(), wd[-1:].clone(), dy)
    large = _ffn(rows, [0, n], [E - 1], wgu, wd, dy)
    for a, b in zip(large[:2], small[:2]):
        _same(a, b)
    for a, b in zip(large[2:], small[2:]):
        _same(a[-1], b[0])
        assert float(a[:-1].abs().max()) == 0.0
