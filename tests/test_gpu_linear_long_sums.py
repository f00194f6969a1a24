"""Long sums on the tensor cores, which cut every addition: the shortfall of sums of one sign, in products whose summed extent is
not split over several tiles.

A group of values that the tensor cores add by themselves takes one addition for 16 of them, each cut by at most 2^-23 of the
running sum, which is half of the group's on average: (values / 16) 2^-24 of the sum."""
import pytest
import torch

import dense_util as D

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def _positive(rows, columns, seed):
    """bf16 values from 1 to 4: a factor a column, so that the sums are spread over a step of bf16."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.rand((rows, columns), generator=g, device="cuda", dtype=BF16).add_(1.0)
    return t.mul_(torch.exp2(torch.rand((columns,), generator=g, device="cuda")).to(BF16))


def _short(got, ref):
    return float(((got.double() - ref) / ref).mean())


def test_weight_gradient_of_many_tokens_is_not_too_small():
    """131072 tokens, 192 tiles (k is not split). 8192 values at a time are added by the tensor cores: at most 3.1e-5 short. The bf16
    rounding is taken out by comparing with the rounded sum: what is left is the mean over 65536 results of how many cross a border."""
    import paper_2609_36959_b200 as cb
    T, K, N = 131072, 4096, 2560
    x, dy = _positive(T, K, 1), _positive(T, N, 2)
    gw = torch.empty((N, K), dtype=BF16, device="cuda")
    cb.linear_backward(dy, x, None, torch.empty(cb.linear_workspace_bytes(T, K, N), dtype=torch.uint8, device="cuda"), grad_w=gw)
    some_n, some_k = torch.arange(0, N, 10, device="cuda"), torch.arange(3, K, 16, device="cuda")
    ref = torch.zeros((len(some_n), len(some_k)), dtype=D.F64, device="cuda")
    for a in range(0, T, 16384):
        ref += dy[a:a + 16384, some_n].double().t() @ x[a:a + 16384, some_k].double()
    got = gw[some_n][:, some_k]
    assert ((got.double() - ref).abs() <= (D.HALF[BF16] * 1.001 + 1e-4) * ref).all()
    short = float(((got.double() - ref.to(BF16).double()) / ref).mean())
    assert abs(short) <= 3.1e-5, short
    assert cb.read_and_clear_device_error() == 0


@pytest.mark.parametrize("T,K,N", [(20003, 264, 136), (8200, 1032, 72), (70001, 8, 8), (300001, 264, 136), (1 << 20, 24, 8), (9000, 4104, 2824)])
def test_weight_gradient_of_long_splits(T, K, N):
    """Sizes that fill no tile, every element against 64 bits: k split into parts below and above 8192 tokens, and (the last) not split.  A part
    adds at most 8192 values at a time."""
    import paper_2609_36959_b200 as cb
    x, dy = _positive(T, K, 3), _positive(T, N, 4)
    whole = torch.full((N + 1, K), 7.0, dtype=BF16, device="cuda")
    cb.linear_backward(dy, x, None, torch.empty(cb.linear_workspace_bytes(T, K, N), dtype=torch.uint8, device="cuda"), grad_w=whole[:N])
    ref = torch.zeros((N, K), dtype=D.F64, device="cuda")
    for a in range(0, T, 1 << 16):
        ref += dy[a:a + (1 << 16)].double().t() @ x[a:a + (1 << 16)].double()
    assert ((whole[:N].double() - ref).abs() <= (D.HALF[BF16] * 1.001 + 6.2e-5) * ref).all() and (whole[N] == 7).all()
    assert cb.read_and_clear_device_error() == 0


def test_fp32_results_are_added_in_pieces():
    """A router's logits, 209 tiles (k is not split), 7168 values: 512 at a time are 1.9e-6 short at most, all at once would be about
    1.3e-5. The sums of the pieces are rounded, not cut: below 14 u = 8.3e-7 each, and far less in the mean."""
    import paper_2609_36959_b200 as cb
    T, K, N = 40001, 7168, 256
    x, w = _positive(T, K, 5), _positive(N, K, 6)
    out = torch.empty((T, N), device="cuda")
    ws = torch.empty(cb.linear_workspace_bytes(T, K, N), dtype=torch.uint8, device="cuda")
    cb.linear(x, w, out, ws)
    for rows in (slice(0, 2000), slice(20000, 22000), slice(T - 2000, T)):
        ref = x[rows].double() @ w.double().t()
        assert abs(_short(out[rows], ref)) <= 2e-6, _short(out[rows], ref)
    # signs that alternate at random: the errors of a sum's pieces are independent, 448 groups of 16 terms cut by 2 u of a running sum
    # no larger than three times the result's rms, 32 at a time: 2 u * 3 * sqrt(32) = 2.0e-6 for all of a piece's, added over 14 pieces
    # of 1 / sqrt(14) the size
    g = torch.Generator(device="cuda").manual_seed(7)
    x.mul_(torch.randint(0, 2, (T, K), generator=g, device="cuda", dtype=torch.int8).mul_(2).sub_(1).to(BF16))
    cb.linear(x, w, out, ws)
    for rows in (slice(0, 2000), slice(T - 2000, T)):
        ref = x[rows].double() @ w.double().t()
        assert float((out[rows].double() - ref).norm() / ref.norm()) <= 2.0e-6
    assert cb.read_and_clear_device_error() == 0
