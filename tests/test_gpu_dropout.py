"""Dropout from the counter: the mask equals the generator's on the CPU bit for bit, and the values equal the
fp32 product and sum of the formula, rounded once."""
import pytest
import torch

import layer_util as L

pytestmark = pytest.mark.gpu


def _want(x, r, p, seed):
    keep, scale = L.dropout_keep(x.numel(), p, seed)
    k = torch.tensor(keep, dtype=torch.bool).reshape(x.shape)
    # one fp32 product and one fp32 sum; a contraction of the two would differ by half a unit of the product
    v = torch.where(k, x.cpu().float() * torch.tensor(scale, dtype=torch.float32), torch.zeros(()))
    return (v if r is None else r.cpu().float() + v), k


def _close(got, want, x, scale):
    half = 2 * L.ULP16 if got.dtype == torch.bfloat16 else 2 * L.ULP32
    err = (got.cpu().double() - want.double()).abs()
    assert (err <= half * want.double().abs() + 2 * L.ULP32 * scale * x.cpu().double().abs()).all(), float(err.max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,p,seed", [(1, 0.5, 1), (7, 0.5, 2), (8, 0.5, 3), (9, 0.1, 2**64 - 1), (1000, 0.25, 12345678901234567890),
                                      (4099, 0.9, 7), (2056, 0.0, 7), (2056, 1.0, 7), (263, 0.999, 5)])
def test_dropout_against_the_formula(n, p, seed, dtype):
    import paper_2609_36959_b200 as cb
    x, r = torch.randn(n, device="cuda").to(dtype), torch.randn(n, device="cuda").to(dtype)
    out, grad = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    alone = torch.full_like(x, 7.0)
    cb.dropout_add(x, r, p, seed, out)
    cb.dropout_add(x, None, p, seed, alone)
    cb.dropout_add_backward(x, p, seed, grad)
    torch.cuda.synchronize()
    _, scale = L.dropout_keep(8, p, seed)
    want, keep = _want(x, r, p, seed)
    _close(out, want, x, scale)
    want, _ = _want(x, None, p, seed)
    _close(alone, want, x, scale)
    assert torch.equal(grad, alone)                        # the adjoint of a diagonal map is itself
    assert torch.equal((alone != 0).cpu(), keep & (x != 0).cpu())


def test_dropout_rate_independence_and_dropped_infinities():
    import paper_2609_36959_b200 as cb
    n = 1 << 20
    one = torch.ones(n, device="cuda")
    a, b = torch.empty_like(one), torch.empty_like(one)
    cb.dropout_add(one, None, 0.25, 11, a)
    cb.dropout_add(one, None, 0.25, 12, b)
    ka, kb = (a != 0).double(), (b != 0).double()
    # five standard deviations of a binomial share of n, and of the share of both
    assert abs(float(ka.mean()) - 0.75) < 5 * (0.75 * 0.25 / n) ** 0.5
    assert abs(float((ka * kb).mean()) - 0.5625) < 5 * (0.5625 * 0.4375 / n) ** 0.5
    assert abs(float((ka[1:] * ka[:-1]).mean()) - 0.5625) < 5 * (2 * 0.5625 * 0.4375 / n) ** 0.5
    bad = torch.full((64,), float("inf"), device="cuda")
    bad[1::2] = float("nan")
    r = torch.randn(64, device="cuda")
    out = torch.empty_like(r)
    cb.dropout_add(bad, r, 1.0, 5, out)
    assert torch.equal(out, r)


def test_dropout_in_place_device_seed_graph_and_stream():
    import paper_2609_36959_b200 as cb
    x, r = torch.randn(33, 1000, device="cuda").to(torch.bfloat16), torch.randn(33, 1000, device="cuda").to(torch.bfloat16)
    want = [torch.empty_like(x) for _ in range(2)]
    for i, seed in enumerate((5, 2**63 + 9)):
        cb.dropout_add(x, r, 0.3, seed, want[i])
    seed_dev = torch.tensor([5], dtype=torch.int64, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(x)
    with torch.cuda.stream(side):
        cb.dropout_add(x, r, 0.3, seed_dev, out)
    side.synchronize()
    assert torch.equal(out, want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cb.dropout_add(x, r, 0.3, seed_dev, out)
    seed_dev.fill_(2**63 + 9 - 2**64)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want[1])
    xi, ri = x.clone(), r.clone()
    cb.dropout_add(xi, r, 0.3, 5, xi)
    cb.dropout_add(x, ri, 0.3, 5, ri)
    assert torch.equal(xi, want[0]) and torch.equal(ri, want[0])


def test_dropout_counter_passes_32_bits():
    """Blocks above 2^32 take the counter's second word: 2^35 elements do not fit, so the generator alone is checked
    against the CPU at such blocks through its definition."""
    low, _ = L.dropout_keep(64, 0.5, 3, first_block=1)
    high, _ = L.dropout_keep(64, 0.5, 3, first_block=(1 << 32) + 1)
    assert low != high
