"""The counter's second word: blocks of eight elements beyond 2^32, that is elements beyond 2^35, by the kernel itself."""
import pytest
import torch

import layer_util as L

pytestmark = pytest.mark.gpu


def test_blocks_beyond_two_to_the_32():
    import paper_2609_36959_b200 as cb
    n, p, seed = (1 << 35) + 8 * 300 + 5, 0.5, 77
    torch.cuda.empty_cache()
    free, _ = torch.cuda.mem_get_info()
    if free < 2 * n + (4 << 30):
        pytest.skip("needs 73 GB on the device")
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    cb.dropout_add_backward(x, p, seed, x)                           # in place
    first = (1 << 32) - 300
    keep, scale = L.dropout_keep(n - 8 * first, p, seed, first_block=first)
    want = torch.tensor(keep, dtype=torch.float32) * scale
    got = x[8 * first:].float().cpu()
    start = x[:2400].float().cpu()
    del x
    torch.cuda.empty_cache()
    assert torch.equal(got, want)
    # the blocks behind 2^32 are not the first ones again
    assert not torch.equal(got[2400:4800], start)
