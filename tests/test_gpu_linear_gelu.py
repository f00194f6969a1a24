"""gelu and its slope over their whole range, negative tails included, against the 64-bit forms.

Pre-activations are exact: one product of two bf16 values each.  With T(a) the normal distribution's tail at a = |v| and u = 2^-24:
the exponent a^2 / 2 takes three roundings (the square, the constant, their product), so that exp(-a^2 / 2) is off by 1.5 a^2 u and
the exponential's own 4 u; the reciprocal (2 u), the approximation (1e-7, below 2 u), the polynomial (two roundings a term, a
condition of at most 1.9 near the ends of its range where the first terms decide: 12 u) and two products (2 u) add 22 u: T to
(1.5 a^2 + 24) u.
gelu is max(v, 0) - a T, one rounding more of either term.  The slope is T or 1 - T plus v phi(v), whose exponential is the same; its T
comes from an approximation good to 1.5e-7 / 2, whose distance from T is also at most 2.2e-4 of the slope for |v| above 2 (both computed in
64 bits over 0 .. 28)."""
import math

import pytest
import torch

import dense_util as D

pytestmark = pytest.mark.gpu
U, BF16 = D.U, torch.bfloat16


def _products(T):
    """x [T, 8], w [64, 8] with one value a row each, and their products [T, 64]: T magnitudes from 2^-10 to 6.4 of both signs,
    times 1 + n / 128."""
    size = torch.exp(torch.linspace(math.log(2.0 ** -10), math.log(6.4), max((T + 1) // 2, 1), dtype=torch.float64, device="cuda"))
    a = torch.cat([-size.flip(0), size])[:T] if T > 1 else torch.tensor([-4.25], dtype=torch.float64, device="cuda")
    a = a.to(BF16)
    b = (1 + torch.arange(64, device="cuda") / 128).to(BF16)
    x, w = torch.zeros((T, 8), dtype=BF16, device="cuda"), torch.zeros((64, 8), dtype=BF16, device="cuda")
    x[:, 3], w[:, 3] = a, b
    return x, w, a.double()[:, None] * b.double()[None]


def _tail(v):
    return 0.5 * torch.special.erfc(v.abs() / math.sqrt(2))


@pytest.mark.parametrize("out_type,residual", [(torch.float32, False), (BF16, False), (BF16, True)])
@pytest.mark.parametrize("T", [1, 3, 4000])
def test_gelu_to_its_own_last_bits(T, out_type, residual):
    import paper_2609_36959_b200 as cb
    x, w, v = _products(T)
    out = torch.empty((T, 64), dtype=out_type, device="cuda")
    ws = torch.empty(cb.linear_workspace_bytes(T, 8, 64), dtype=torch.uint8, device="cuda")
    cb.linear(x, w, out, ws, act="gelu", residual=torch.zeros_like(out) if residual else None)
    tail = v.abs() * _tail(v)
    ref = v.clamp_min(0) - tail
    tol = (1.5 * v * v + 25) * U * tail + U * ref.abs() + 2.0 ** -126
    if out_type == BF16:
        tol = tol + D.HALF[BF16] * (ref.abs() + tol)
    worst = ((out.double() - ref).abs() / tol).max()
    assert worst <= 1, float(worst)


@pytest.mark.parametrize("T", [1, 4000])
def test_gelu_slope_to_its_own_last_bits(T):
    """The pre-activation is given as the forward call would have kept it, in bf16."""
    import paper_2609_36959_b200 as cb
    x, w, v = _products(T)
    pre = v.to(BF16)
    v = pre.double()
    ws = torch.empty(cb.linear_workspace_bytes(T, 8, 64), dtype=torch.uint8, device="cuda")
    dy, d, gx = torch.ones((T, 64), dtype=BF16, device="cuda"), torch.empty((T, 64), dtype=BF16, device="cuda"), torch.empty_like(x)
    cb.linear_backward(dy, None, w, ws, act="gelu", pre=pre, grad_pre=d, grad_x=gx)
    tail, bump = _tail(v), v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
    ref = torch.where(v > 0, 1 - tail, tail) + bump
    tol = (1.5 * v * v + 25) * U * (tail + bump.abs()) + 2 * U * (v > 0) + 2.0 ** -126
    tol = tol + torch.where(v.abs() > 2, 2.2e-4 * ref.abs(), torch.full_like(ref, 7.6e-8)).clamp_max(7.6e-8)
    tol = tol + D.HALF[BF16] * (ref.abs() + tol)
    worst = ((d.double() - ref).abs() / tol).max()
    assert worst <= 1, float(worst)


def test_gelu_at_the_ends_of_the_range():
    """Infinities, NaN, zeros of both signs and values whose tail is below the range."""
    import paper_2609_36959_b200 as cb
    for T in (1, 40):
        bias = torch.tensor([math.inf, -math.inf, math.nan, 0.0, -0.0, 1e30, -1e30, -20.0], device="cuda").to(BF16)
        out = torch.empty((T, 8), device="cuda")
        ws = torch.empty(cb.linear_workspace_bytes(T, 8, 8), dtype=torch.uint8, device="cuda")
        cb.linear(torch.zeros((T, 8), dtype=BF16, device="cuda"), torch.zeros((8, 8), dtype=BF16, device="cuda"), out, ws, bias=bias, act="gelu")
        assert torch.isposinf(out[:, 0]).all() and (out[:, [1, 3, 4, 6, 7]] == 0).all() and torch.isnan(out[:, 2]).all()
        assert (out[:, 5] == bias[5].float()).all()
