"""NaN logits wherever they stand, expert 0 among them: chosen first in ascending id, ids distinct and in range."""
import math

import pytest
import torch

import layer_util as L

pytestmark = pytest.mark.gpu


def _gate(logits, K, sigmoid):
    import paper_2609_36959_b200 as cb
    T, E = logits.shape
    ids = torch.full((T, K), -9, dtype=torch.int32, device="cuda")
    w = torch.full((T, K), 7.0, device="cuda")
    cb.gate_topk(logits, ids, w, flags=cb.GATE_SIGMOID if sigmoid else 0)
    torch.cuda.synchronize()
    assert cb.read_and_clear_device_error() == 0
    return ids, w


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("E,K", [(1, 1), (8, 2), (8, 8), (16, 16), (33, 9), (100, 3), (256, 8), (1000, 16), (1024, 16)])
def test_nan_is_chosen_first(E, K, dtype, sigmoid):
    g = torch.Generator().manual_seed(E + K)
    rows = (torch.randn((9, E), generator=g) * 2).to(dtype)
    nan = math.nan
    rows[0, 0] = nan                                     # expert 0 alone
    rows[1, :] = nan                                     # all of them
    rows[2, 0] = rows[2, E - 1] = nan                    # the first and the last
    rows[3, E // 2] = nan
    rows[4, :] = math.inf                                # NaN is above +inf
    rows[4, 0] = nan
    rows[5, :] = -math.inf
    rows[5, 0] = nan
    rows[6, : min(E, 4)] = nan
    rows[7, 0] = -torch.tensor(nan)                      # with its sign bit set
    ids, w = _gate(rows.cuda(), K, sigmoid)              # row 8 has no NaN
    want, _, _ = L.gate_forward(rows, K, sigmoid)
    # among NaN the plain form's order is by id too (stable sort)
    assert torch.equal(ids.cpu().long(), want)
    for r in ids.tolist():
        assert len(set(r)) == K and min(r) >= 0 and max(r) < E
    assert bool(torch.isnan(w[:8]).all()) and bool(torch.isfinite(w[8]).all())
