"""Layers that share one object's buffers, with parameters of their own."""
import pytest
import torch

import test_gpu_moe_layer_dense as dense
import workloads as W

pytestmark = pytest.mark.gpu


def test_layers_that_share_an_objects_buffers():
    """Two layers' parameters take turns in one object, as its documentation says; results are those of an object each."""
    w = W.make_custom(90, 8, 2, 64, 2, 2, 3, seed=11, C=2)
    names = ("gamma", "w_router", "b_router", "w_gate_up", "w_down", "w_shared_up", "b_shared_up", "w_shared_down", "b_shared_down")
    objects = [dense._layer(w, 72, 136, norm="rms", router="linear", p=0.1) for _ in range(3)]
    shared, x, r, dy = objects[2]
    layers = [o[0] for o in objects[:2]]
    for name in names:                                              # the second layer's parameters are others
        getattr(layers[1], name).mul_(-0.75)
    params = [{name: getattr(m, name) for name in names} for m in layers]
    inputs = [(x, r), (r, x)]

    def gradients(m):
        return [getattr(m, "grad_" + name).clone() for name in names]

    want, kept = [], []
    for m, (a, b) in zip(layers, inputs):
        m.forward(a, 5, residual=b)
        m.restore(m.save())
        want.append([m.backward(dy).clone()] + gradients(m))
    for p, (a, b) in zip(params, inputs):
        for name in names:
            setattr(shared, name, p[name])
        shared.forward(a, 5, residual=b)
        kept.append(shared.save())
    for i in (1, 0):
        for name in names:
            setattr(shared, name, params[i][name])
        shared.restore(kept[i])
        got = [shared.backward(dy).clone()] + gradients(shared)
        assert all(torch.equal(a, b) for a, b in zip(got, want[i]))
