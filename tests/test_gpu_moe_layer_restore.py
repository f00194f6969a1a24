"""What a restored layer's backward pass differentiates."""
import pytest
import torch

import dense_util as D
import test_gpu_moe_layer_dense as dense
import workloads as W

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H", [64, 264])
def test_restored_norm_passes_see_the_same_rows(H):
    """rstd, the normalised rows and the gradients are those of the same values: gamma's gradient is the fp32 sum of grad_n z over
    the restored rows ((T + 64) u sum|grad_n z| and 4 u more), z = rows rstd, with rstd theirs."""
    w = W.make_custom(90, 8, 2, H, 2, 2, 3, seed=11, C=2)
    m, x, r, dy = dense._layer(w, 72, 0, norm="rms", router="plain")
    m.forward(x, dense.SEED, residual=r)
    kept = m.save()
    m.restore(kept)
    m.backward(dy)
    rows = m.x.double()
    rstd = 1 / torch.sqrt((rows * rows).mean(1) + m.eps)
    assert ((m.rstd.double() - rstd).abs() <= 24 * D.U * rstd).all()
    dyz = m.grad_n.double() * rows * m.rstd.double()[:, None]
    assert ((m.grad_gamma.double() - dyz.sum(0)).abs() <= (w.T + 68) * D.U * dyz.abs().sum(0) + 1e-38).all()
    # the rows are the checkpoint's, rounded to the layer's type
    assert torch.equal(m.x, D.values(*kept.rows, 128).float().to(torch.bfloat16))
