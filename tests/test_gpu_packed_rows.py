"""Rows in 8 bits and back against the 64-bit definition.

The codes are exactly the definition's: 16- and 32-bit values divided by one another lie on a border between codes or at
least 2^-33 of themselves away from it, far more than 64 bits are off by.  A scale is the group's largest value times the
rounded 1 / L, rounded (2 u and u^2: 2.01 u), a value one product of two fp32 numbers more, rounded once more to bf16.  The scale of a
group whose largest value is above 3e38 may be one step (2 u) lower, so that L times it stays finite."""
import math

import pytest
import torch

import dense_util as D

pytestmark = pytest.mark.gpu
CODES = [torch.int8, torch.float8_e4m3fn]


def _pack(x, code, group):
    import paper_2609_36959_b200 as cb
    T, H = x.shape
    groups = len(D.groups_of(H, group))
    q = torch.full((T + 1, H), 7, dtype=torch.uint8, device="cuda").view(code)
    scales = torch.full((T + 1, groups), 7.0, device="cuda")
    cb.pack_rows(x, q[:T], scales[:T])
    out = torch.full((T + 1, H), 7.0, dtype=x.dtype, device="cuda")
    cb.unpack_rows(q[:T], scales[:T], out[:T])
    torch.cuda.synchronize()
    assert (q[T].view(torch.uint8) == 7).all() and (scales[T] == 7).all() and (out[T] == 7).all()      # the row behind the last
    return q[:T], scales[:T], out[:T]


def _check(x, code, group, got):
    q, scales, out = got
    rq, rs = D.pack(x, code, group)
    assert torch.equal(q.to(D.F64), rq), int((q.to(D.F64) != rq).sum())
    nan = torch.isnan(rs)
    assert torch.equal(torch.isnan(scales), nan)
    down = 2 * D.U * (rs * D.LARGEST[code] > 3e38)                   # the step at the end of the range
    assert ((scales.double() - rs).abs()[~nan] <= ((2.01 * D.U + down) * rs.abs())[~nan] + 2.0 ** -149).all()
    ref = D.values(rq, rs, group)
    bad = torch.isnan(ref)
    assert torch.equal(torch.isnan(out), bad)
    half = 0 if x.dtype == torch.float32 else D.HALF[x.dtype]
    relative = (3.01 * D.U + half + D.values(torch.ones_like(ref), down, group)) * (1 + 2 * D.U)
    assert ((out.double() - ref).abs()[~bad] <= (relative * ref.abs())[~bad] + 127 * 2.0 ** -149).all()


@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("code", CODES, ids=["i8", "e4m3"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H", [(1, 8), (1, 7168), (3, 24), (5, 128), (7, 136), (700, 264), (9, 1000), (33, 1024), (2000, 512), (5, 4104), (3, 16384)])
def test_pack_against_definition(T, H, dtype, code, group):
    g = torch.Generator(device="cuda").manual_seed(T * 1009 + H)
    x = torch.randn((T, H), generator=g, device="cuda").to(dtype)
    x = (x.float() * torch.exp(3 * torch.randn((T, 1), generator=g, device="cuda"))).to(dtype)
    x[T // 2, : H // 2] = 0                                           # whole groups of zeros among them
    got = _pack(x, code, group)
    _check(x, code, group, got)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, _pack(x, code, group)))


@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("code", CODES, ids=["i8", "e4m3"])
def test_pack_halfway_values(code, group):
    """Groups whose largest value is a power of two, 2, of values k / 64: the int8 quotient 127 k / 128 is halfway where k is 64
    modulo 128 (two of the 257 values of k, about 255 of the 32 768 here), the e4m3 quotient 7 k / 2 at many borders."""
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randint(-128, 129, (64, 512), generator=g, device="cuda").float() / 64
    x[:, ::128] = 2.0
    for dtype in (torch.bfloat16, torch.float32):
        _check(x.to(dtype), code, group, _pack(x.to(dtype), code, group))
    assert int(((x.double() * 127 / 2) % 1 == 0.5).sum()) > 100


@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("code", CODES, ids=["i8", "e4m3"])
def test_pack_extremes(code, group):
    """Infinities and NaN stay in their group, the type's largest values and tiny groups keep their codes."""
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn((12, 384), generator=g, device="cuda")
    x[1, 5], x[2, 200], x[3, 383] = math.inf, math.nan, -math.inf
    x[4] *= 1e-32                                                     # the factor L / most is past 1e30
    x[5] = torch.finfo(torch.float32).max * torch.sign(x[5])
    x[6] *= 1e37
    x[7] = 0
    x[8] = -0.0
    x[10] *= 6e37                                                     # a reciprocal below the normal range
    x[9] *= 2.0 ** -60
    x[9, 0] = 1.0                                                     # everything else in its group far below a step
    _check(x, code, group, _pack(x, code, group))


def test_pack_on_an_odd_boundary_and_in_views():
    """Pointers 16 bytes, not 32, from a boundary take the narrow form and give the same bits."""
    import paper_2609_36959_b200 as cb
    g = torch.Generator(device="cuda").manual_seed(7)
    for dtype, shift in ((torch.bfloat16, 8), (torch.float32, 4)):
        x = torch.randn((40, 256), generator=g, device="cuda").to(dtype)
        room = torch.zeros(40 * 256 + 16, dtype=dtype, device="cuda")
        moved = room[shift:shift + 40 * 256].view(40, 256)
        moved.copy_(x)
        a, b = _pack(x, torch.int8, 128), _pack(moved, torch.int8, 128)
        assert all(torch.equal(u, v) for u, v in zip(a, b))
        out = torch.zeros_like(room)
        cb.unpack_rows(a[0], a[1], out[shift:shift + 40 * 256].view(40, 256))
        assert torch.equal(out[shift:shift + 40 * 256].view(40, 256), a[2])


def test_pack_no_rows():
    import paper_2609_36959_b200 as cb
    x = torch.zeros((0, 64), dtype=torch.bfloat16, device="cuda")
    cb.pack_rows(x, torch.zeros((0, 64), dtype=torch.int8, device="cuda"), torch.zeros((0, 1), device="cuda"))
