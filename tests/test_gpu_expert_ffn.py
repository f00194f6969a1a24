"""The experts' feed-forward block and its gradients against the 64-bit plain form.

Bounds, element by element (h = 2^-9, half a unit of bf16; q = 2^-10, half a unit of the nine-bit mantissa of pre, with
2^-40 where it underflows; u = 2^-24): the kernel rounds act and grad_pre to bf16 and pre to its own 16 bits once each and
accumulates in fp32, so
  act    h |act| + what g and u are off by, (H u) (|x| |W|^T) times the slopes, at most 1.1 |u| and |silu(g)|
  out    sum |d act| |Wd| + F u sum |act| |Wd| + h |out|
  d_pre  d_act is off by H u (|dy| |Wd|); from the rounded g and u: |d_act| (1.1 h |g|) for d_u and
         |d_act| |u| (1.1 h + 0.5 h |g|) for d_g (|silu'| <= 1.1, |silu''| <= 0.5), and the rounding h |d_pre|
  dx, dW the sums of those over the other factor's magnitude, n u of the terms' sum, and h of the result
Every bound is taken twice."""
import pytest
import torch

import layer_util as L

pytestmark = pytest.mark.gpu
h, U = L.ULP16, L.ULP32
q, TINY = 2.0 ** -10, 2.0 ** -40


def _case(seed, counts, experts, E, H, F, lead=0, tail=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def rnd(*s, by=1.0):
        return (torch.randn(s, generator=g, device="cuda") * by).to(torch.bfloat16)

    offsets = [lead]
    for c in counts:
        offsets.append(offsets[-1] + c)
    P = offsets[-1] + tail
    ranges = [(offsets[i], offsets[i + 1], experts[i]) for i in range(len(counts)) if counts[i] and 0 <= experts[i] < E]
    return dict(rows=rnd(P, H, by=scale), dy=rnd(P, H), wgu=rnd(E, 2 * F, H, by=H ** -0.5), wd=rnd(E, H, F, by=F ** -0.5),
                offsets=torch.tensor(offsets, dtype=torch.int32, device="cuda"),
                slots=torch.tensor(experts, dtype=torch.int32, device="cuda"), ranges=ranges, E=E, H=H, F=F, P=P)


def _run(c, backward=True, in_place=False, want=("dx", "dgu", "ddn"), fill=7.0):
    import paper_2609_36959_b200 as cb
    P, E, H, F = c["P"], c["E"], c["H"], c["F"]

    def new(*s):
        return torch.full(s, fill, dtype=torch.bfloat16, device="cuda")

    ws = torch.full((cb.expert_ffn_workspace_bytes(P, len(c["slots"]), E, H, F),), 0xCD, dtype=torch.uint8, device="cuda")
    r = dict(out=new(P, H), act=new(P, F))
    args = (c["offsets"], c["slots"], c["wgu"], c["wd"])
    if backward:
        r.update(pre=new(P, 2 * F), dx=new(P, H), dgu=new(E, 2 * F, H), ddn=new(E, H, F))
        cb.expert_ffn(c["rows"], *args, r["act"], r["out"], ws, pre=r["pre"])
        kept = r["pre"].clone()
        r["d_pre"] = r["pre"] if in_place else new(P, 2 * F)
        cb.expert_ffn_backward(c["dy"], c["rows"], *args, r["pre"], r["act"], r["d_pre"], ws,
                               grad_rows=r["dx"] if "dx" in want else None, grad_w_gate_up=r["dgu"] if "dgu" in want else None,
                               grad_w_down=r["ddn"] if "ddn" in want else None)
        if not in_place:
            assert torch.equal(kept.view(torch.int16), r["pre"].view(torch.int16))
    else:
        cb.expert_ffn(c["rows"], *args, r["act"], r["out"], ws)
    torch.cuda.synchronize()
    return r


def _check(c, r, backward=True):
    import paper_2609_36959_b200 as cb
    assert cb.read_and_clear_device_error() == 0
    H, F = c["H"], c["F"]
    ref, act, pre = L.ffn_forward(c["rows"], c["ranges"], c["wgu"], c["wd"])
    X, DY, WGU, WD = (c[k].double().abs() for k in ("rows", "dy", "wgu", "wd"))
    inside = torch.zeros(c["P"], dtype=torch.bool, device="cuda")
    b = L.ffn_backward(c["dy"], c["rows"], c["ranges"], c["wgu"], c["wd"]) if backward else None
    t_gu, t_dn = torch.zeros_like(WGU), torch.zeros_like(WD)

    def within(name, got, want, tol):
        err = (got.double() - want).abs()
        assert (err <= 2 * tol + 1e-30).all(), (name, float((err - 2 * tol).max()), float(err.max()))

    for a, z, e in c["ranges"]:
        inside[a:z] = True
        off = H * U * (X[a:z] @ WGU[e].t())                    # of g and of u before rounding
        g, u = pre[a:z, :F], pre[a:z, F:]
        silu = (g * torch.sigmoid(g)).abs()
        t_act = h * act[a:z].abs() + 1.1 * u.abs() * off[:, :F] + silu * off[:, F:] + 4 * U * act[a:z].abs()
        within("act", r["act"][a:z], act[a:z], t_act)
        within("out", r["out"][a:z], ref[a:z], t_act @ WD[e].t() + F * U * (act[a:z].abs() @ WD[e].t()) + h * ref[a:z].abs())
        if not backward:
            continue
        within("pre", L.decode_pre(r["pre"][a:z]) if r["pre"] is not r["d_pre"] else pre[a:z], pre[a:z], off + q * pre[a:z].abs() + TINY)
        da = b["d_act"][a:z].abs()
        off_da = H * U * (DY[a:z] @ WD[e])
        og, ou = off[:, :F] + q * g.abs() + TINY, off[:, F:] + q * u.abs() + TINY
        t_g = off_da * 1.1 * u.abs() + da * (1.1 * ou + 0.5 * u.abs() * og) + h * b["d_pre"][a:z, :F].abs()
        t_u = off_da * silu + da * 1.1 * og + h * b["d_pre"][a:z, F:].abs()
        t = torch.cat([t_g, t_u], 1)
        within("d_pre", r["d_pre"][a:z], b["d_pre"][a:z], t)
        d = b["d_pre"][a:z].abs()
        within("dx", r["dx"][a:z], b["dx"][a:z], t @ WGU[e] + 2 * F * U * (d @ WGU[e]) + h * b["dx"][a:z].abs())
        t_gu[e] += t.t() @ X[a:z] + c["P"] * U * (d.t() @ X[a:z])
        t_dn[e] += DY[a:z].t() @ t_act + c["P"] * U * (DY[a:z].t() @ act[a:z].abs())
    for name in ("out", "act") + (("dx",) if backward else ()):
        assert (r[name][~inside] == 7.0).all(), name                # rows of no slot are not written
    if backward:
        within("dgu", r["dgu"], b["dgu"], t_gu + h * b["dgu"].abs())
        within("ddn", r["ddn"], b["ddn"], t_dn + h * b["ddn"].abs())


SHAPES = [
    # counts of the slots, experts of the slots, E, H, F
    ([1], [0], 1, 8, 8),
    ([1], [0], 1, 64, 64),
    ([3, 0, 5], [1, 0, 1], 2, 72, 40),
    ([1, 1, 1, 1, 1, 1], [0, 1, 2, 3, 4, 5], 8, 128, 96),
    ([17, 128, 1, 0, 64], [2, 0, 2, 1, 3], 4, 136, 200),
    ([33, 31, 129, 255], [0, 1, 0, 1], 2, 256, 128),
    ([257, 256, 300], [1, -1, 0], 2, 192, 320),
    ([600, 5, 0, 200], [0, 2, 1, 0], 3, 520, 264),
    ([70, 70], [0, 0], 1, 1024, 1408),
    ([0, 0], [0, 1], 2, 64, 64),
    ([1000], [0], 1, 2048, 512),
]


@pytest.mark.parametrize("counts,experts,E,H,F", SHAPES)
def test_expert_ffn_against_plain(counts, experts, E, H, F):
    counts = [0 if e < 0 else n for n, e in zip(counts, experts)]
    c = _case(H + F, counts, experts, E, H, F)
    r = _run(c)
    _check(c, r)
    r2 = _run(c)
    for k in r:                                                       # the same bits every time
        assert torch.equal(r[k].view(torch.int16), r2[k].view(torch.int16)), k
    alone = _run(c, backward=False)
    for k in ("out", "act"):
        assert torch.equal(alone[k].view(torch.int16), r[k].view(torch.int16))


@pytest.mark.parametrize("P", [1, 2, 7, 8, 9, 16])
@pytest.mark.parametrize("H,F", [(8, 8), (264, 200), (2048, 1408), (1032, 16)])
def test_a_few_rows(P, H, F):
    """Calls of one row up to the size where tiles take over, rows outside the slots and bad slots among them."""
    import paper_2609_36959_b200 as cb
    counts = [0, 1, 0, P - 1, 0]
    c = _case(P + H, counts, [2, 0, 1, 3, -1], 4, H, F, lead=0, tail=0)
    _check(c, _run(c))
    both = _case(P + F, [P // 2, P - P // 2], [1, 1], 2, H, F)      # replicas of one expert
    _check(both, _run(both))
    if P > 2:
        c = _case(P, [1, P - 2], [0, 1], 2, H, F, lead=1)
        _check(c, _run(c))
        good = _run(c)
        c["slots"] = torch.tensor([0, 7], dtype=torch.int32, device="cuda")
        r = _run(c, backward=False)
        assert cb.read_and_clear_device_error() == cb.DEVERR_BAD_SLOT
        assert torch.equal(r["out"][1:2], good["out"][1:2]) and (r["out"][2:] == 7.0).all()


def test_rows_outside_the_slots_stay_untouched():
    c = _case(5, [40, 0, 3, 130], [1, 0, 2, 0], 3, 128, 64, lead=13, tail=21)
    _check(c, _run(c))


def test_many_ragged_slots():
    g = torch.Generator().manual_seed(1)
    counts = torch.randint(0, 40, (200,), generator=g).tolist()
    experts = torch.randint(0, 50, (200,), generator=g).tolist()
    c = _case(9, counts, experts, 50, 264, 72)
    _check(c, _run(c))


def test_in_place_gradient_and_single_outputs():
    c = _case(6, [30, 200, 1], [0, 1, 0], 2, 136, 72)
    r = _run(c)
    _check(c, r)
    p = _run(c, in_place=True)
    for k in ("out", "d_pre", "dx", "dgu", "ddn"):
        assert torch.equal(p[k].view(torch.int16), r[k].view(torch.int16)), k
    for one in ("dx", "dgu", "ddn"):
        s = _run(c, want=(one,))
        assert torch.equal(s[one].view(torch.int16), r[one].view(torch.int16))
        for other in ("dx", "dgu", "ddn"):
            assert other == one or (s[other] == 7.0).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_non_finite_rows_stay_in_their_slot(bad):
    """Slots end inside tiles: a neighbour's NaN or infinity must not reach another slot's rows or weights."""
    c = _case(7, [37, 50, 70], [0, 1, 2], 3, 136, 136)
    clean = _run(c)
    c["rows"][37:87] = bad
    c["dy"][37:87] = bad
    r = _run(c)
    for k in ("out", "dx", "act", "pre", "d_pre"):
        for a, b in ((0, 37), (87, 157)):
            assert torch.equal(r[k][a:b].view(torch.int16), clean[k][a:b].view(torch.int16)), k
    for k in ("dgu", "ddn"):
        for e in (0, 2):
            assert torch.equal(r[k][e].view(torch.int16), clean[k][e].view(torch.int16)), k
        assert not torch.isfinite(r[k][1].float()).any()
    # non-finite weights of one expert stay with that expert
    c = _case(7, [37, 50, 70], [0, 1, 2], 3, 136, 136)
    c["wgu"][1], c["wd"][1] = bad, bad
    r = _run(c)
    for k in ("out", "dx"):
        for a, b in ((0, 37), (87, 157)):
            assert torch.equal(r[k][a:b].view(torch.int16), clean[k][a:b].view(torch.int16)), k


@pytest.mark.parametrize("P", [3, 40])
def test_saved_preactivations_over_their_range(P):
    """Values from below the finest code to above the largest: nearest codes, gradual underflow, saturation, NaN kept."""
    import paper_2609_36959_b200 as cb
    H = F = 8
    scale = [2.0 ** e for e in (-45, -39, -30, 0, 20, 31, 40, 100)]
    rows = torch.zeros((P, H), dtype=torch.bfloat16, device="cuda")
    for i in range(P):
        rows[i, i % H] = 1.0 + (i % 5) * 0.375
    wgu = torch.zeros((1, 2 * F, H), dtype=torch.bfloat16, device="cuda")
    for f in range(2 * F):
        for k in range(H):
            wgu[0, f, k] = scale[(f + k) % 8] * (1 if f % 2 else -1)
    wgu[0, 3, 1] = float("nan")
    act, out, pre = (torch.full((P, n), 7.0, dtype=torch.bfloat16, device="cuda") for n in (F, H, 2 * F))
    ws = torch.empty(cb.expert_ffn_workspace_bytes(P, 1, 1, H, F), dtype=torch.uint8, device="cuda")
    cb.expert_ffn(rows, torch.tensor([0, P], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), wgu,
                  torch.zeros((1, H, F), dtype=torch.bfloat16, device="cuda"), act, out, ws, pre=pre)
    got = L.decode_pre(pre)
    want = torch.stack([wgu[0].double() @ rows[i].double() for i in range(P)])
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan)
    most = 2.0 ** 31 * (1 + 511 / 512)
    want = want.clamp(-most, most)
    assert ((got - want)[~nan].abs() <= (q * want.abs() + TINY)[~nan]).all()


def test_large_gates_saturate_without_nan():
    c = _case(8, [64, 9], [0, 1], 2, 128, 64, scale=100.0)       # |g| in the hundreds: exp(-g) overflows
    r = _run(c)
    _check(c, r)
    assert torch.isfinite(r["out"].float()).all() and torch.isfinite(r["dx"].float()).all()


def test_bad_offsets_and_slots_are_flagged_and_skipped():
    import paper_2609_36959_b200 as cb
    c = _case(3, [20, 30, 10], [0, 1, 0], 2, 64, 64)
    good = _run(c)
    c["slots"] = torch.tensor([0, 5, 0], dtype=torch.int32, device="cuda")
    r = _run(c)
    assert cb.read_and_clear_device_error() == cb.DEVERR_BAD_SLOT
    for a, b in ((0, 20), (50, 60)):
        assert torch.equal(r["out"][a:b], good["out"][a:b])
    assert (r["out"][20:50] == 7.0).all()
    c["slots"] = torch.tensor([0, 1, 0], dtype=torch.int32, device="cuda")
    c["offsets"] = torch.tensor([0, 20, 10, 100000], dtype=torch.int32, device="cuda")   # decreases, then past P
    r = _run(c)
    assert cb.read_and_clear_device_error() == cb.DEVERR_BAD_SLOT
    assert torch.equal(r["out"][:10], good["out"][:10])


def test_no_rows_at_all_and_another_stream():
    import paper_2609_36959_b200 as cb
    c = _case(4, [0, 0], [0, 1], 2, 64, 64)
    r = _run(c)
    assert float(r["dgu"].float().abs().sum()) == 0 and float(r["ddn"].float().abs().sum()) == 0
    c = _case(4, [100, 60], [0, 1], 2, 128, 72)
    want = _run(c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _run(c)
    for k in want:
        assert torch.equal(want[k].view(torch.int16), got[k].view(torch.int16)), k
    assert cb.read_and_clear_device_error() == 0


def test_gradient_against_differences():
    """Directional derivatives of the 64-bit loss against the kernel's bf16 gradients: each gradient is off by at most
    its bound above, about 2 % of its terms' magnitudes at these sizes."""
    c = _case(11, [40, 25, 13], [0, 1, 0], 2, 64, 48)
    r = _run(c)
    dy = c["dy"].double()
    g = torch.Generator(device="cuda").manual_seed(8)

    def loss(x, a, b):
        return float((L.ffn_forward(x, c["ranges"], a, b)[0] * dy).sum())

    base = [c["rows"].double(), c["wgu"].double(), c["wd"].double()]
    for i, grad in enumerate((r["dx"], r["dgu"], r["ddn"])):
        v = torch.randn(base[i].shape, generator=g, device="cuda", dtype=torch.float64)
        up, down = list(base), list(base)
        up[i], down[i] = base[i] + 1e-5 * v, base[i] - 1e-5 * v
        num = (loss(*up) - loss(*down)) / 2e-5
        terms = grad.double() * v
        assert abs(num - float(terms.sum())) <= 0.02 * float(terms.abs().sum())
