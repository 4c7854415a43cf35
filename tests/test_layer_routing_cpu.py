"""A layer that was trained with a routing of its own carries it, and the calls that
route by the softmax over the kept logits refuse the layer (CPU only)."""

import os

import numpy as np
import pytest
import torch

from paper_2609_21137_amd import fit, synth


@pytest.fixture(scope="module")
def C():
    from paper_2609_21137_amd import build
    if not os.path.exists(build.LIB):
        build.build()
    from paper_2609_21137_amd import cardan
    return cardan


def _layer():
    return synth.make_layer(128, 64, 6, 4, 16, 8, 5)


def _trained(routing, L=None, **kw):
    L = L or _layer()
    return fit.TrainedLayer(L, 2, 4, device="cpu", routing=routing, **kw).layer(L)


@pytest.mark.parametrize("routing", [dict(score="sigmoid"), dict(renorm=False), dict(scale=2.5), dict(groups=3, top_groups=2),
                                     dict(score="sigmoid", groups=3, top_groups=2, group_best=2, scale=0.5)])
def test_routing_stays_with_the_layer(routing):
    out = _trained(routing)
    assert out["routing"] == routing
    again = fit.TrainedLayer(out, 2, 4, device="cpu")
    assert again.routing == routing and again.layer(out)["routing"] == routing
    # another one takes its place, the layer's own leaves none
    assert _trained(dict(scale=3.0), out)["routing"] == dict(scale=3.0)
    assert "routing" not in _trained({}, out) and "routing" in out


def test_bias_stays_with_the_layer(C):
    bias = torch.linspace(-1, 1, 6)
    out = _trained(dict(bias=bias))
    assert set(out["routing"]) == {"bias"} and out["routing"]["bias"].dtype == np.float32
    assert np.array_equal(out["routing"]["bias"], bias.numpy())
    assert torch.equal(fit.TrainedLayer(out, 2, 4, device="cpu").routing["bias"], bias)
    assert torch.equal(C.DeviceLayer.from_numpy(out, "cpu").routing["bias"], bias)


@pytest.mark.parametrize("routing", [None, {}, dict(score="softmax", renorm=True, scale=1.0, bias=None),
                                     dict(groups=3, top_groups=3, group_best=2)])
@pytest.mark.parametrize("router", [False, True])
def test_a_layers_own_routing_leaves_nothing(C, routing, router):
    out = _trained(routing, train_router=router)
    assert "routing" not in out and C.DeviceLayer.from_numpy(out, "cpu").routing is None


def test_calls_that_route_refuse_it(C):
    shape, x = C.make_shape(128, 64, 6, 2, 4, 16, 8), torch.zeros(1, 128, dtype=torch.bfloat16)
    layer = C.DeviceLayer.from_numpy(_trained(dict(score="sigmoid")), "cpu")
    W_down = torch.zeros(6, 64, 128, dtype=torch.bfloat16)
    for call in (lambda: C.moe_layer(shape, x, layer), lambda: C.moe_layer_relu2(shape, x, layer),
                 lambda: C.moe_layer_noalloc(shape, x, layer), lambda: C.moe_decode_step(shape, x, [layer, layer]),
                 lambda: C.moe_layer_dense_down(shape, x, layer, W_down)):
        with pytest.raises(ValueError, match="routing of its own"):
            call()
    # given a routing, it is no matter (and the tensors are looked at)
    with pytest.raises(ValueError, match="GPU"):
        C.vq_lr_expert_ffn(shape, x, torch.zeros(1, 2).int(), torch.zeros(1, 2), torch.zeros(2, 1, 8), layer)
