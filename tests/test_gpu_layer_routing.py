"""A layer distilled with a routing of its own, run as it is documented: route_rows
by the layer's routing, then the experts. Against the trained layer's forward pass,
which rounds the experts' matrices, their activations and their outputs to bf16
(2^-8 each, and the logits' selection is the same): 3 percent in the 2-norm."""

import numpy as np
import pytest
import torch
from test_gpu_distill_fit import _setup

from paper_2609_21137_amd import fit

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def C():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_21137_amd import cardan
    return cardan


@pytest.mark.parametrize("router", [False, True])
@pytest.mark.parametrize("routing", [dict(score="sigmoid", scale=2.5, groups=3, top_groups=2, group_best=2), dict(renorm=False),
                                     dict(score="sigmoid", bias=True)])
def test_distilled_layer_runs_by_its_routing(C, routing, router):
    L, k, d, x, head, teacher, ids, labels = _setup("silu_glu", 8, False)
    routing = dict(routing)
    if "bias" in routing:
        routing["bias"] = torch.linspace(-0.5, 0.5, 6, device="cuda")
    out, history = fit.distill_layer(L, x, head, teacher, ids, k, d, labels=labels, steps=2, rows=40, lr=1e-3,
                                     optimizer="adamw", routing=routing, train_router=router)
    assert np.isfinite(history).all()
    layer = C.DeviceLayer.from_numpy(out)
    shape, t = C.make_shape(128, 64, 6, k, d, 16, 8), layer.tensors
    with pytest.raises(ValueError):
        C.moe_layer(shape, x[:1].contiguous(), layer)
    student = fit.TrainedLayer(out, k, d)
    for B in (1, 3, 64):
        xb = x[:B].contiguous()
        logits = xb.double() @ t["router_w"].double() + t["router_bias"].double()
        idx, w, _, _ = C.route_rows(logits, k, **layer.routing)
        y = C.vq_lr_expert_ffn(shape, xb, idx, w, C.shared_proj(shape, xb, t["U_gate"], t["U_up"]), layer)
        want = student.forward(xb)
        assert torch.equal(student.route(xb)[0], idx.long())
        assert float((y - want).norm() / want.norm()) <= 0.03
