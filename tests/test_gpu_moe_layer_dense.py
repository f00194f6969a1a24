"""A layer with the root-mean-square norm, the residual added in it, 32-bit logits and a dense block beside the experts, against
the 64-bit chain with the gradients of autograd; the layer's input kept in 8 bits and restored; the dense block in 8 bits.

The chain rounds about a dozen intermediate tensors to bf16, each by at most 2^-8 of its size, 2^-8 / sqrt 3 in the 2-norm, and the
block's pre-activation to int8 codes: half a step of largest / 127 at most, 0.65 % of a normal value's size in the 2-norm (largest
about 2.8 of them in 128), which its slope passes on with a factor below 0.5.  12 * 2^-8 / sqrt 3 + 0.4 % is 3.1 % if all errors
pointed one way; 3 % are allowed.  The choice of experts is taken from the layer (it is discrete, and tested by itself)."""
import pytest
import torch

import dense_util as D
import layer_util as L
import workloads as W

pytestmark = pytest.mark.gpu
SEED = 2**40 + 17


def _layer(w, F, shared, **more):
    import paper_2609_36959_b200 as cb
    from paper_2609_36959_b200.moe import MoELayer
    layout = cb.Layout(w.N, w.Q, w.S, w.E, w.slot_expert.tolist(), w.primary_slot.tolist())
    m = MoELayer(layout, w.slot_expert.tolist(), w.T, w.K, w.H, F, shared=shared, **more)
    g = torch.Generator(device="cuda").manual_seed(4)

    def rnd(*s):
        return torch.randn(s, generator=g, device="cuda")

    m.step.src_rank.copy_(torch.from_numpy(w.src_rank))
    m.gamma.copy_(1 + 0.2 * rnd(w.H))
    for name, scale in (("w_router", w.H ** -0.5), ("b_router", 0.2), ("w_gate_up", w.H ** -0.5), ("w_down", F ** -0.5), ("w_shared_up", w.H ** -0.5),
                        ("b_shared_up", 0.2), ("w_shared_down", max(shared, 1) ** -0.5), ("b_shared_down", 0.2)):
        if hasattr(m, name):
            t = getattr(m, name)
            t.copy_(rnd(*t.shape) * scale)
    x, r, dy = (rnd(w.T, w.H).to(torch.bfloat16) for _ in range(3))
    return m, x, r, dy


def _chain(m, rows, seed):
    """out from the rows that the norm takes, and the leaves, in 64 bits."""
    names = ("gamma", "w_router", "b_router", "w_gate_up", "w_down", "w_shared_up", "b_shared_up", "w_shared_down", "b_shared_down")
    leaf = {k: getattr(m, k).detach().double().requires_grad_() for k in names if hasattr(m, k)}
    leaf["rows"] = rows.detach().double().requires_grad_()
    s = leaf["rows"]
    n = s / torch.sqrt((s * s).mean(1, keepdim=True) + m.eps) * leaf["gamma"]
    ids = m.step.topk_ids.long()
    logits = n @ leaf["w_router"].t()
    if "b_router" in leaf:
        logits = logits + leaf["b_router"]
    weight = torch.softmax(logits.gather(1, ids), 1)
    y = torch.zeros_like(n)
    for e in range(m.E):
        t, k = torch.nonzero(ids == e, as_tuple=True)
        g, u = n[t] @ leaf["w_gate_up"][e, :m.F].t(), n[t] @ leaf["w_gate_up"][e, m.F:].t()
        y = y.index_add(0, t, (g * torch.sigmoid(g) * u) @ leaf["w_down"][e].t() * weight[t, k][:, None])
    keep, scale = L.dropout_keep(s.numel(), m.p, seed)
    out = s + torch.tensor(keep, dtype=torch.float64, device="cuda").reshape(s.shape) * scale * y
    if m.shared:
        out = out + D.act(n @ leaf["w_shared_up"].t() + leaf["b_shared_up"], m.shared_act) @ leaf["w_shared_down"].t() + leaf["b_shared_down"]
    return out, leaf


def _near(name, got, want):
    off = float((got.double() - want).norm()) / float(want.norm())
    assert off <= 0.03, (name, off)


def _check_gradients(m, gx, leaf):
    _near("x", gx, leaf["rows"].grad)
    for name in leaf:
        if name != "rows":
            _near(name, getattr(m, "grad_" + name), leaf[name].grad)


@pytest.mark.parametrize("T,K,shared,act,router,p", [(96, 2, 136, "silu", "linear", 0.1), (70, 3, 0, "silu", "linear", 0.0), (3, 2, 64, "gelu", "plain", 0.25),
                                                     (300, 2, 200, "relu", "linear", 0.0)])
def test_layer_against_the_chain_in_64_bits(T, K, shared, act, router, p):
    import paper_2609_36959_b200 as cb
    w = W.make_custom(T, 8, K, 64, 2, 2, 3, seed=21, C=2)
    m, x, r, dy = _layer(w, 72, shared, norm="rms", router=router, shared_act=act, p=p)
    out = m.forward(x, SEED, residual=r).clone()
    gx = m.backward(dy).clone()
    torch.cuda.synchronize()
    assert cb.read_and_clear_device_error() == 0
    rows = (x.double() + r.double()).to(torch.bfloat16)
    assert torch.equal(m.x, rows)
    ref, leaf = _chain(m, rows, SEED)
    ref.backward(dy.double())
    _near("out", out, ref.detach())
    _check_gradients(m, gx, leaf)
    # again, and from a gradient that the layer returned
    assert torch.equal(m.backward(dy), gx)
    again = m.backward(gx).clone()
    assert torch.equal(m.backward(m.grad_x.copy_(gx)), again)


@pytest.mark.parametrize("norm,shared,p", [("rms", 136, 0.1), ("layer", 0, 0.0), ("rms", 0, 0.25)])
def test_restored_layer(norm, shared, p):
    """Two layers share the buffers: after the other one's forward call, restore gives the gradients at the rows that were kept."""
    import paper_2609_36959_b200 as cb
    w = W.make_custom(90, 8, 2, 264, 2, 2, 3, seed=11, C=2)
    m, x, r, dy = _layer(w, 72, shared, norm=norm, router="linear" if shared else "plain", p=p)
    if norm == "rms":
        out = m.forward(x, SEED, residual=r).clone()
    else:
        m.beta.copy_(0.1 * torch.randn(w.H, device="cuda"))
        out = m.forward(x, SEED).clone()
    plain = m.backward(dy).clone()
    kept, ids, offsets = m.save(), m.step.topk_ids.clone(), m.step.dest_offsets.clone()
    m.step.src_rank.zero_()
    m.forward((2 * x.float() + 1).to(torch.bfloat16), SEED + 1)         # another layer's tokens over everything
    m.restore(kept)
    gx = m.backward(dy).clone()
    torch.cuda.synchronize()
    assert cb.read_and_clear_device_error() == 0
    assert torch.equal(m.step.topk_ids, ids) and torch.equal(m.step.dest_offsets, offsets)
    if norm == "rms":
        ref, leaf = _chain(m, D.values(*kept.rows, 128), SEED)
        ref.backward(dy.double())
        _check_gradients(m, gx, leaf)
    # rows that are off by 0.65 % change the gradient by about as much (its own roundings are of that size): within 3 %
    _near("as without", gx, plain.double())
    assert torch.isfinite(out.float()).all()


def test_dense_block_in_8_bits():
    """The block on the operands that the layer quantised, in 64 bits: hidden rows and result to half a step of bf16 (and the fp32
    sums of 64 and 144 products)."""
    import paper_2609_36959_b200 as cb
    for norm in ("rms", "layer"):
        w = W.make_custom(50, 8, 2, 64, 2, 2, 3, seed=3, C=2)
        m, x, r, _ = _layer(w, 40, 144, norm=norm, shared_8bit=True)
        m.pack_shared()
        out = m.forward(x, 5, residual=r) if norm == "rms" else m.forward(x, 5)
        torch.cuda.synchronize()
        assert cb.read_and_clear_device_error() == 0
        n, up = D.values(*m.n8, 0), D.values(*m.w_shared_up8, 0)
        hidden = D.act(n @ up.t() + m.b_shared_up.double(), "silu")
        assert ((m.shared_hidden.double() - hidden).abs() <= 2.0 ** -8 * hidden.abs() + 64 * 2.0 ** -22 * (n.abs() @ up.abs().t()) + 2.0 ** -18).all()
        h8, down = D.values(*m.shared_hidden8, 0), D.values(*m.w_shared_down8, 0)
        base = h8 @ down.t() + m.b_shared_down.double() + m.x.double()
        assert ((m.base.double() - base).abs() <= 2.0 ** -8 * base.abs() + 144 * 2.0 ** -22 * (h8.abs() @ down.abs().t()) + 2.0 ** -18).all()
        assert torch.equal(out, (m.step.y.float() + m.base.float()).to(torch.bfloat16))
        # the codes are those of the norm's rows: e4m3 to half a step
        ref = m.step.x.double()
        assert ((n - ref).abs() <= (2.0 ** -4 + 2.0 ** -8) * ref.abs() + 2.0 ** -10 * m.n8[1].double()).all()
        with pytest.raises(cb.CobaltError):
            m.backward(x)


def test_layer_without_tokens():
    import paper_2609_36959_b200 as cb
    w = W.make_custom(0, 8, 2, 64, 2, 2, 3, seed=3, C=2)
    m, x, r, dy = _layer(w, 40, 136, norm="rms", router="linear")
    for t in (m.grad_w_shared_up, m.grad_b_shared_down, m.grad_w_router, m.grad_gamma):
        t.fill_(3.0)
    out = m.forward(x, 1, residual=r)
    m.restore(m.save())
    assert out.shape == m.backward(dy).shape == (0, 64)
    torch.cuda.synchronize()
    assert cb.read_and_clear_device_error() == 0
    for t in (m.grad_w_shared_up, m.grad_b_shared_down, m.grad_w_router, m.grad_gamma):
        assert (t == 0).all()


def test_layer_refusals():
    import paper_2609_36959_b200 as cb
    w = W.make_custom(8, 8, 2, 64, 2, 2, 3, seed=3, C=2)
    for bad in (dict(norm="batch"), dict(router="none"), dict(shared=12), dict(shared=24, shared_8bit=True), dict(shared=16, shared_act="tanh")):
        with pytest.raises(ValueError):
            _layer(w, 40, bad.pop("shared", 0), **bad)
    m, x, r, _ = _layer(w, 40, 0)
    with pytest.raises(cb.CobaltError):
        m.save()
    with pytest.raises(cb.CobaltError):
        m.forward(x, 1, residual=r)


def test_layer_in_a_graph():
    """Forward and backward captured once and replayed with other inputs give what the plain calls give."""
    import paper_2609_36959_b200 as cb
    for T in (3, 300):
        w = W.make_custom(T, 8, 2, 64, 2, 2, 3, seed=5, C=2)
        m, x, r, dy = _layer(w, 72, 136, norm="rms", router="linear", p=0.2)
        fixed = x.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(2):
                m.forward(fixed, 9, residual=r)
                m.backward(dy)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            m.forward(fixed, 9, residual=r)
            m.backward(dy)
        names = ("out", "grad_x", "grad_w_shared_up", "grad_w_shared_down", "grad_b_router", "grad_gamma", "grad_w_router")
        for seed in (1, 2):
            g = torch.Generator(device="cuda").manual_seed(seed)
            other = torch.randn(x.shape, generator=g, device="cuda").to(torch.bfloat16)
            fixed.copy_(other)
            graph.replay()
            got = [getattr(m, k).clone() for k in names]
            m.forward(other, 9, residual=r)
            m.backward(dy)
            torch.cuda.synchronize()
            for a, k in zip(got, names):
                assert torch.equal(a, getattr(m, k)), k
        assert cb.read_and_clear_device_error() == 0
