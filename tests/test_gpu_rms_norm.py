"""Root-mean-square norm of a sum, its 8-bit output and its gradients against the 64-bit plain form.

Bounds (u = 2^-24): the sum of a row's squares is at most 32 additions in a thread and ten levels of a tree, all of one
sign: 42 u relative; rstd half of that and two units of the root: 24 u; y two products more: 26 u, then half a step of the result's
type.  The mean of g z is a sum of signed terms: 48 u mean|g z|.  grad_gamma is an fp32 sum over T rows in any order:
(T + 64) u sum|dy z| and what z is off by."""
import math

import pytest
import torch

import dense_util as D

pytestmark = pytest.mark.gpu
U = D.U
SIZES = [(1, 8), (1, 7168), (3, 24), (5, 256), (700, 264), (33, 512), (9, 1000), (2000, 1024), (17, 1032), (300, 4096), (5, 8192), (6, 8200), (3, 16384)]


def _inputs(T, H, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def rnd(*s):
        return torch.randn(s, generator=g, device="cuda")

    x, r, dy, ds = ((rnd(T, H) * c).to(dtype) for c in (2.0, 3.0, 1.0, 0.5))
    return x, r, dy, ds, rnd(H) * 0.3 + 1


def _check_backward(dy, s, gamma, rstd, ds, dx, dg, dtype):
    """s: the rows' values in 64 bits; rstd as the kernel was given it."""
    T = dy.shape[0]
    ref, rg = D.rms_backward(dy, s, gamma, rstd.double()[:, None], ds)
    z, rs, dyd = s * rstd.double()[:, None], rstd.double()[:, None], dy.double()
    g = (dyd * gamma.double()).abs()
    mean = (g * z.abs()).mean(1, keepdim=True)
    tol = 64 * U * rs * (g + z.abs() * mean) + (0 if ds is None else 4 * U * ds.double().abs()) + D.HALF[dtype] * ref.abs() * (1 + 64 * U) + 1e-38
    assert ((dx.double() - ref).abs() <= tol).all(), float(((dx.double() - ref).abs() - tol).max())
    tol = (T + 64) * U * (dyd * z).abs().sum(0) + 4 * U * (dyd * z).abs().sum(0) + 1e-38
    assert ((dg.double() - rg).abs() <= tol).all()


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H", SIZES)
def test_rms_norm_against_plain(T, H, dtype, residual):
    import paper_2609_36959_b200 as cb
    x, r, dy, ds, gamma = _inputs(T, H, dtype, T * 100003 + H)
    r, ds = (r, ds) if residual else (None, None)

    def run():
        total, y, dx = (torch.full((T + 1, H), 7.0, dtype=dtype, device="cuda") for _ in range(3))
        rstd, dg = torch.full((T,), 7.0, device="cuda"), torch.full((H,), 7.0, device="cuda")
        ws = torch.full((cb.rms_norm_workspace_bytes(T, H),), 0xAB, dtype=torch.uint8, device="cuda")
        cb.rms_norm(x, gamma, 1e-5, residual=r, sum_out=total[:T] if residual else None, y=y[:T], rstd=rstd)
        s = total[:T] if residual else x
        cb.rms_norm_backward(dy, s, gamma, rstd, dx[:T], dg, ws, grad_sum=ds)
        torch.cuda.synchronize()
        assert (y[T] == 7).all() and (dx[T] == 7).all() and (not residual or (total[T] == 7).all())
        return s, y[:T], rstd, dx[:T], dg

    got = run()
    s, y, rstd, dx, dg = got
    if residual:
        assert torch.equal(s, (x.double() + r.double()).to(dtype))
    ref, rs = D.rms_forward(s, gamma, 1e-5)
    assert ((rstd.double() - rs[:, 0]).abs() <= 24 * U * rs[:, 0]).all()
    assert ((y.double() - ref).abs() <= (26 * U + D.HALF[dtype]) * (1 + 32 * U) * ref.abs() + 1e-38).all()
    _check_backward(dy, s.double(), gamma, rstd, ds, dx, dg, dtype)
    assert all(torch.equal(a, b) for a, b in zip(got, run()))          # the same bits every time


@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("code", [torch.float8_e4m3fn, torch.int8], ids=["e4m3", "i8"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H", [(1, 8), (1, 7168), (5, 264), (700, 512), (9, 1000), (17, 1032), (40, 4096), (3, 16384)])
def test_rms_norm_in_8_bits(T, H, dtype, code, group):
    """A code is off by half a step of its own, and a little more where y's rounding (28 u with the factor's) moves a value over a
    border: int8 (1/2 + 127 * 64 u) scales, e4m3 2^-4 (1 + 64 u) of the value or half the smallest step."""
    import paper_2609_36959_b200 as cb
    x, r, _, _, gamma = _inputs(T, H, dtype, T * 7 + H)
    q = torch.full((T + 1, H), 7, dtype=torch.uint8, device="cuda").view(code)
    scales = torch.full((T + 1, len(D.groups_of(H, group))), 7.0, device="cuda")
    total, y = torch.empty_like(x), torch.empty_like(x)
    cb.rms_norm(x, gamma, 1e-5, residual=r, sum_out=total, packed=(q[:T], scales[:T]))
    torch.cuda.synchronize()
    assert (q[T].view(torch.uint8) == 7).all() and (scales[T] == 7).all()
    ref, _ = D.rms_forward(total, gamma, 1e-5)
    _, rs = D.pack(ref, code, group)
    assert ((scales[:T].double() - rs).abs() <= 32 * U * rs).all()
    got, step = D.values(q[:T], scales[:T], group), D.values(torch.ones_like(ref), scales[:T], group)
    if code == torch.int8:
        tol = (0.5 + 127 * 64 * U) * step
    else:
        tol = torch.maximum(2.0 ** -4 * (1 + 64 * U) * ref.abs(), 2.0 ** -10 * (1 + 64 * U) * step)
    assert ((got - ref).abs() <= tol + 64 * U * ref.abs()).all()
    # with y, and without the sum: the same codes
    q2, scales2 = torch.zeros_like(q), torch.zeros_like(scales)
    cb.rms_norm(x, gamma, 1e-5, residual=r, y=y, packed=(q2[:T], scales2[:T]))
    assert torch.equal(q2[:T].view(torch.uint8), q[:T].view(torch.uint8)) and torch.equal(scales2[:T], scales[:T])
    assert ((y.double() - ref).abs() <= (26 * U + D.HALF[dtype]) * (1 + 32 * U) * ref.abs() + 1e-38).all()


@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("code", [torch.int8, torch.float8_e4m3fn], ids=["i8", "e4m3"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H", [(1, 8), (700, 264), (9, 1000), (300, 1032), (64, 4096), (5, 7168), (3, 16384)])
def test_rms_norm_backward_from_8_bits(T, H, dtype, code, group):
    """The gradients at the rows that were kept: as of rows of those values."""
    import paper_2609_36959_b200 as cb
    x, _, dy, ds, gamma = _inputs(T, H, dtype, T * 13 + H)
    q = torch.empty((T, H), dtype=torch.uint8, device="cuda").view(code)
    scales = torch.empty((T, len(D.groups_of(H, group))), device="cuda")
    rstd, dx, dg = torch.empty(T, device="cuda"), torch.empty_like(x), torch.empty(H, device="cuda")
    y, ws = torch.empty_like(x), torch.empty(cb.rms_norm_workspace_bytes(T, H), dtype=torch.uint8, device="cuda")
    cb.rms_norm(x, gamma, 1e-5, y=y, rstd=rstd)
    cb.pack_rows(x, q, scales)
    for grad_sum in (None, ds):
        cb.rms_norm_backward(dy, (q, scales), gamma, rstd, dx, dg, ws, grad_sum=grad_sum)
        torch.cuda.synchronize()
        _check_backward(dy, D.values(q, scales, group), gamma, rstd, grad_sum, dx, dg, dtype)


def test_rms_norm_in_place():
    import paper_2609_36959_b200 as cb
    x, r, dy, ds, gamma = _inputs(50, 2048, torch.bfloat16, 3)
    total, y = torch.empty_like(x), torch.empty_like(x)
    rstd, dx, dg = torch.empty(50, device="cuda"), torch.empty_like(x), torch.empty(2048, device="cuda")
    ws = torch.empty(cb.rms_norm_workspace_bytes(50, 2048), dtype=torch.uint8, device="cuda")
    cb.rms_norm(x, gamma, 1e-5, residual=r, sum_out=total, y=y, rstd=rstd)
    cb.rms_norm_backward(dy, total, gamma, rstd, dx, dg, ws, grad_sum=ds)
    x2, r2, dy2, ds2 = x.clone(), r.clone(), dy.clone(), ds.clone()
    cb.rms_norm(x2, gamma, 1e-5, residual=r2, sum_out=r2, y=x2, rstd=rstd)      # the stream in its place, y over x
    assert torch.equal(r2, total) and torch.equal(x2, y)
    cb.rms_norm_backward(dy2, total, gamma, rstd, dy2, dg, ws, grad_sum=ds)
    cb.rms_norm_backward(dy, total, gamma, rstd, ds2, dg, ws, grad_sum=ds2)
    assert torch.equal(dy2, dx) and torch.equal(ds2, dx)


def test_rms_norm_odd_rows():
    """Rows with a NaN, an infinity, zeros and huge values: what the formulas give, in their own rows only."""
    import paper_2609_36959_b200 as cb
    x, _, dy, _, gamma = _inputs(8, 640, torch.float32, 4)
    x[1, 3], x[2, 5], x[3], x[4] = math.nan, math.inf, 0.0, 1e30        # 1e30 squared overflows: rstd 0
    y, rstd = torch.empty_like(x), torch.empty(8, device="cuda")
    q, scales = torch.empty((8, 640), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty((8, 1), device="cuda")
    cb.rms_norm(x, gamma, 1e-5, y=y, rstd=rstd, packed=(q, scales))
    torch.cuda.synchronize()
    assert torch.isnan(y[1]).all() and torch.isnan(y[2, 5]) and (y[2, :5] == 0).all() and (y[3] == 0).all() and (y[4] == 0).all()
    assert torch.isnan(scales[1]) and torch.isnan(scales[2]) and scales[3] == 0 and (q[1:5].float() == 0).all()
    ref, _ = D.rms_forward(x, gamma, 1e-5)
    keep = [0, 5, 6, 7]
    assert ((y.double() - ref)[keep].abs() <= 28 * U * ref[keep].abs()).all()
    dx, dg = torch.empty_like(x), torch.empty(640, device="cuda")
    ws = torch.empty(cb.rms_norm_workspace_bytes(8, 640), dtype=torch.uint8, device="cuda")
    cb.rms_norm_backward(dy, x, gamma, rstd, dx, dg, ws)
    torch.cuda.synchronize()
    assert torch.isnan(dx[1]).all() and torch.isfinite(dx[[0, 3, 4, 5, 6, 7]]).all()


def test_rms_norm_no_rows():
    import paper_2609_36959_b200 as cb
    x = torch.empty((0, 64), device="cuda")
    rstd, dg = torch.empty(0, device="cuda"), torch.full((64,), 7.0, device="cuda")
    ws = torch.empty(cb.rms_norm_workspace_bytes(0, 64), dtype=torch.uint8, device="cuda")
    cb.rms_norm(x, torch.ones(64, device="cuda"), 1e-5, y=x, rstd=rstd)
    cb.rms_norm_backward(x, x, torch.ones(64, device="cuda"), rstd, x, dg, ws)
    torch.cuda.synchronize()
    assert (dg == 0).all()


@pytest.mark.parametrize("code", [torch.int8, torch.float8_e4m3fn], ids=["i8", "e4m3"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rms_norm_in_8_bits_of_the_smallest_values(dtype, code):
    """Rows so small that L / most is past the range, zeros among them.  x is a multiple of 2^-133 and gamma 1, so that s gamma is exact;
    y is good to 26 u, a code's product to 4 u more, and the scale, below 2^-126, to 2^-150: 448 2^-150 of a value."""
    import paper_2609_36959_b200 as cb
    for H, group in ((264, 128), (264, 0), (4096, 128), (4096, 0)):
        g = torch.Generator(device="cuda").manual_seed(H)
        x = (torch.randint(-9, 10, (5, H), generator=g, device="cuda").double() * 2.0 ** -133).to(dtype)
        x[0, 1:] = 0
        q, scales = torch.empty(x.shape, dtype=code, device="cuda"), torch.empty((5, len(D.groups_of(H, group))), device="cuda")
        cb.rms_norm(x, torch.ones(H, device="cuda"), 1e-5, packed=(q, scales))
        ref, _ = D.rms_forward(x, torch.ones(H, device="cuda"), 1e-5)
        got, step = D.values(q, scales, group), D.values(torch.ones_like(ref), scales, group)
        half = 0.5 * step if code == torch.int8 else torch.maximum(2.0 ** -4 * ref.abs(), 2.0 ** -10 * step)
        assert ((got - ref).abs() <= half * (1 + 64 * U) + 64 * U * ref.abs() + 448 * 2.0 ** -150).all()


@pytest.mark.parametrize("second", [False, True])
@pytest.mark.parametrize("rows", ["plain", "i8", "e4m3"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H", [(1300, 5120), (700, 8192), (450, 16384)])
def test_rms_norm_gradients_of_several_long_rows_a_cta(T, H, dtype, rows, second):
    """Every CTA has more than one row, so that the next one's loads are under way; and the result takes the gradient's place."""
    import paper_2609_36959_b200 as cb
    x, _, dy, ds, gamma = _inputs(T, H, dtype, T + H)
    s, kept = x.double(), x
    if rows != "plain":
        kept = torch.empty((T, H), dtype=torch.int8 if rows == "i8" else torch.float8_e4m3fn, device="cuda"), torch.empty((T, H // 128), device="cuda")
        cb.pack_rows(x, *kept)
        s = D.values(*kept, 128)
    rstd = (1.0 / torch.sqrt((s * s).mean(1) + 1e-5)).float()
    ws = torch.full((cb.rms_norm_workspace_bytes(T, H),), 0xAB, dtype=torch.uint8, device="cuda")
    dx, dg = dy.clone(), torch.empty(H, device="cuda")
    cb.rms_norm_backward(dx, kept, gamma, rstd, dx, dg, ws, grad_sum=ds if second else None)
    _check_backward(dy, s, gamma, rstd, ds if second else None, dx, dg, dtype)


@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("code", [torch.int8, torch.float8_e4m3fn], ids=["i8", "e4m3"])
def test_rms_norm_in_8_bits_of_infinities_and_nan(code, group):
    """A NaN makes its row's values NaN.  An infinity makes rstd 0: its own group's values are NaN, the row's other groups 0."""
    import paper_2609_36959_b200 as cb
    x, _, _, _, gamma = _inputs(4, 512, torch.bfloat16, 9)
    x[1, 200], x[2, 300] = float("nan"), float("inf")
    x[3] = 0
    q, scales = torch.full((4, 512), 7, dtype=torch.uint8, device="cuda").view(code), torch.zeros((4, len(D.groups_of(512, group))), device="cuda")
    y = torch.empty_like(x)
    cb.rms_norm(x, gamma, 1e-5, y=y, packed=(q, scales))
    v = D.values(q, scales, group)
    assert torch.isnan(v[1]).all() and torch.isnan(y[1]).all() and (q[1].view(torch.uint8) == 0).all()
    bad = torch.isnan(v[2])
    want = torch.zeros_like(bad)
    want[256:384] = True
    assert bad.all() if group == 0 else torch.equal(bad, want) and (v[2][~want] == 0).all()
    assert torch.isnan(y[2, 300]) and (v[3] == 0).all() and torch.isfinite(v[0]).all()
