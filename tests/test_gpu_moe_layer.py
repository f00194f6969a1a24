"""A whole layer, norm to residual, against the 64-bit chain with the gradients of autograd.

The layer rounds about ten intermediate tensors to bf16, each by at most 2^-9 of its size, and the chain's factors are of
order one at these sizes: outputs and gradients agree to 10 * 2^-9, about 2 %, in the 2-norm; 3 % are allowed.  The choice
of experts is taken from the layer (it is discrete, and tested by itself)."""
import pytest
import torch

import layer_util as L
import workloads as W

pytestmark = pytest.mark.gpu


def _layer(w, F, gate, p):
    import paper_2609_36959_b200 as cb
    from paper_2609_36959_b200.moe import MoELayer
    layout = cb.Layout(w.N, w.Q, w.S, w.E, w.slot_expert.tolist(), w.primary_slot.tolist())
    m = MoELayer(layout, w.slot_expert.tolist(), w.T, w.K, w.H, F, gate=gate, p=p)
    g = torch.Generator(device="cuda").manual_seed(4)
    m.step.src_rank.copy_(torch.from_numpy(w.src_rank))
    m.gamma.copy_(1 + 0.2 * torch.randn(w.H, generator=g, device="cuda"))
    m.beta.copy_(0.1 * torch.randn(w.H, generator=g, device="cuda"))
    for t, scale in ((m.w_router, w.H ** -0.5), (m.w_gate_up, w.H ** -0.5), (m.w_down, F ** -0.5)):
        t.copy_(torch.randn(t.shape, generator=g, device="cuda") * scale)
    x = (torch.randn((w.T, w.H), generator=g, device="cuda") + 0.3).to(torch.bfloat16)
    dy = torch.randn((w.T, w.H), generator=g, device="cuda").to(torch.bfloat16)
    return m, x, dy


def _chain(m, x, seed, sigmoid):
    """out and the leaves, in 64 bits."""
    leaf = {k: v.detach().double().requires_grad_() for k, v in dict(x=x, gamma=m.gamma, beta=m.beta, w_router=m.w_router,
                                                                     w_gate_up=m.w_gate_up, w_down=m.w_down).items()}
    xx = leaf["x"]
    mu = xx.mean(1, keepdim=True)
    n = (xx - mu) / torch.sqrt(((xx - mu) ** 2).mean(1, keepdim=True) + m.eps) * leaf["gamma"] + leaf["beta"]
    ids = m.step.topk_ids.long()
    chosen = (n @ leaf["w_router"].t()).gather(1, ids)
    score = torch.sigmoid(chosen) if sigmoid else torch.softmax(chosen, 1)
    weight = score / score.sum(1, keepdim=True)
    y = torch.zeros_like(n)
    for e in range(m.E):
        t, k = torch.nonzero(ids == e, as_tuple=True)
        g, u = n[t] @ leaf["w_gate_up"][e, :m.F].t(), n[t] @ leaf["w_gate_up"][e, m.F:].t()
        y = y.index_add(0, t, (g * torch.sigmoid(g) * u) @ leaf["w_down"][e].t() * weight[t, k][:, None])
    keep, scale = L.dropout_keep(x.numel(), m.p, seed)
    mask = torch.tensor(keep, dtype=torch.float64, device="cuda").reshape(x.shape) * scale
    return xx + mask * y, leaf


@pytest.mark.parametrize("gate,p,T,K", [("softmax", 0.0, 96, 2), ("sigmoid", 0.25, 70, 3), ("softmax", 0.1, 1, 2)])
def test_layer_against_the_chain_in_64_bits(gate, p, T, K):
    import paper_2609_36959_b200 as cb
    w = W.make_custom(T, 8, K, 64, 2, 2, 3, seed=21, C=2)
    m, x, dy = _layer(w, 72, gate, p)
    seed = 2**40 + 17
    out = m.forward(x, seed).clone()
    gx = m.backward(dy).clone()
    torch.cuda.synchronize()
    assert cb.read_and_clear_device_error() == 0
    ref, leaf = _chain(m, x, seed, gate == "sigmoid")
    ref.backward(dy.double())

    def near(name, got, want):
        off = float((got.double() - want).norm()) / float(want.norm())
        assert off <= 0.03, (name, off)

    near("out", out, ref.detach())
    near("x", gx, leaf["x"].grad)
    for name in ("gamma", "beta", "w_router", "w_gate_up", "w_down"):
        near(name, getattr(m, "grad_" + name), leaf[name].grad)


def test_layer_repeats_and_follows_its_stream():
    w = W.make_custom(50, 8, 2, 64, 2, 2, 3, seed=3, C=2)
    m, x, dy = _layer(w, 40, "softmax", 0.2)
    out, gx = m.forward(x, 5).clone(), m.backward(dy).clone()
    kept = m.grad_w_gate_up.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out2, gx2 = m.forward(x, 5).clone(), m.backward(dy).clone()
    side.synchronize()
    assert torch.equal(out.view(torch.int16), out2.view(torch.int16)) and torch.equal(gx.view(torch.int16), gx2.view(torch.int16))
    assert torch.equal(kept.view(torch.int16), m.grad_w_gate_up.view(torch.int16))
    assert not torch.equal(m.forward(x, 6), out)


def test_layer_in_a_graph():
    """Forward and backward captured once and replayed with other inputs give what the plain calls give."""
    import paper_2609_36959_b200 as cb
    for T in (3, 300):                                   # a few rows, and tiles
        w = W.make_custom(T, 8, 2, 64, 2, 2, 3, seed=5, C=2)
        m, x, dy = _layer(w, 72, "softmax", 0.2)
        fixed = x.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(2):
                m.forward(fixed, 9)
                m.backward(dy)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            m.forward(fixed, 9)
            m.backward(dy)
        for seed in (1, 2, 3):
            g = torch.Generator(device="cuda").manual_seed(seed)
            other = torch.randn(x.shape, generator=g, device="cuda").to(torch.bfloat16)
            fixed.copy_(other)
            graph.replay()
            got = [t.clone() for t in (m.out, m.grad_x, m.grad_w_gate_up, m.grad_w_down, m.grad_gamma)]
            want_out = m.forward(other, 9).clone()
            want = [want_out, m.backward(dy).clone(), m.grad_w_gate_up, m.grad_w_down, m.grad_gamma]
            torch.cuda.synchronize()
            for a, b in zip(got, want):
                assert torch.equal(a.view(torch.int16), b.view(torch.int16))
        assert cb.read_and_clear_device_error() == 0
