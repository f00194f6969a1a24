"""Offsets that decrease or pass P: flagged, read as their running maximum, every row written by its own slot alone, and
nothing written behind the workspace."""
import pytest
import torch

pytestmark = pytest.mark.gpu
GUARD = 1 << 16


def _run(offsets, slots, data, F, guard=True):
    import paper_2609_36959_b200 as cb
    rows, dy, wgu, wd = data
    (P, H), E, D = rows.shape, wd.shape[0], len(slots)

    def new(*s):
        return torch.full(s, 7.0, dtype=torch.bfloat16, device="cuda")

    n = cb.expert_ffn_workspace_bytes(P, D, E, H, F)
    room = torch.full((n + GUARD,), 0xCD, dtype=torch.uint8, device="cuda")
    off = torch.tensor([o - 2**32 if o >= 2**31 else o for o in offsets], dtype=torch.int32, device="cuda")
    slot = torch.tensor(slots, dtype=torch.int32, device="cuda")
    act, out, pre, dx, dgu, ddn = new(P, F), new(P, H), new(P, 2 * F), new(P, H), new(E, 2 * F, H), new(E, H, F)
    cb.expert_ffn(rows, off, slot, wgu, wd, act, out, room[:n], pre=pre)
    kept = pre.clone()
    # in place: a row that two tiles took would be read after it was overwritten
    cb.expert_ffn_backward(dy, rows, off, slot, wgu, wd, pre, act, pre, room[:n], grad_rows=dx, grad_w_gate_up=dgu, grad_w_down=ddn)
    torch.cuda.synchronize()
    flagged = cb.read_and_clear_device_error()
    assert bool((room[n:] == 0xCD).all())
    return flagged, dict(act=act, out=out, pre=kept, d_pre=pre, dx=dx, dgu=dgu, ddn=ddn)


def _running(offsets, P):
    top, r = 0, []
    for i, o in enumerate(offsets):
        top = min(o, P) if i == 0 else max(top, min(o, P))
        r.append(top)
    return r


@pytest.mark.parametrize("P,offsets,slots", [
    (4096, [(0, 4096)[i & 1] for i in range(65)], [i % 3 for i in range(64)]),
    (6000, [0, 6000, 0, 6000, 0], [0, 1, 2, 0]),
    (6000, [100, 3000, 2000, 5000, 1, 5900, 6000], [0, 1, 2, 1, 0, 2]),
    (700, [50, 650, 0, 80, 700], [0, 1, 2, 1]),
    (700, [0, 300, 200, 2**32 - 1, 5], [0, 1, 2, 1]),
    (700, [0, 300, 200, 500, 700], [0, -1, 9, 1]),
    (8, [(0, 8)[i & 1] for i in range(65)], [i % 3 for i in range(64)]),
    (8, [5, 8, 0, 4, 7], [0, 1, 2, 1]),
    (7, [1, 4, 2, 6, 2**31 + 5], [0, 1, 2, 1]),
    (6, [0, 3, 1, 5, 6], [0, -1, 9, 1]),
])
def test_offsets_out_of_order(P, offsets, slots):
    import paper_2609_36959_b200 as cb
    E, H, F = 3, 72, 40
    g = torch.Generator(device="cuda").manual_seed(P)

    def rnd(*s):
        return torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)

    data = rnd(P, H), rnd(P, H), rnd(E, 2 * F, H), rnd(E, H, F)
    flagged, got = _run(offsets, slots, data, F)
    assert flagged == cb.DEVERR_BAD_SLOT
    in_order = _running(offsets, P)
    # the same rows by offsets that are in order, without the slots that hold no expert
    holds = [e if 0 <= e < E and in_order[d + 1] > in_order[d] else -1 for d, e in enumerate(slots)]
    flagged, want = _run(in_order, holds, data, F)
    skipped = any(h < 0 and in_order[d + 1] > in_order[d] for d, h in enumerate(holds))
    assert flagged == (cb.DEVERR_BAD_SLOT if skipped else 0)
    for k in got:
        assert torch.equal(got[k].view(torch.int16), want[k].view(torch.int16)), k
    written = torch.zeros(P, dtype=torch.bool, device="cuda")
    for d, e in enumerate(holds):
        if e >= 0:
            written[in_order[d]:in_order[d + 1]] = True
    assert bool((got["out"][~written] == 7.0).all()) and bool((got["out"][written] != 7.0).any(1).all())
