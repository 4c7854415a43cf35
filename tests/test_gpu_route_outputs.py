"""What route_rows returns are tensors of their own: calls that ask for 16-byte
alignment take them at every size, and a change of one is no change of another."""

import pytest
import torch

from paper_2609_21137_amd import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def C():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_21137_amd import cardan
    return cardan


@pytest.mark.parametrize("N,k", [(1, 7), (3, 5), (1, 1), (7, 3), (2, 4), (64, 7)])
def test_a_layers_experts_take_the_routing(C, N, k):
    """route_rows, then the experts for that routing: as with aligned copies of it, and, the routing
    being the layer's own, as the whole layer (its weights are within 2^-22 of these; y within 1e-5)."""
    H, I, E, d, K, r = 128, 64, 8, 4, 16, 8
    L = C.DeviceLayer.from_numpy(synth.make_layer(H, I, E, d, K, r, 5))
    shape = C.make_shape(H, I, E, k, d, K, r)
    g = torch.Generator(device="cuda").manual_seed(N)
    x = torch.randn((N, H), generator=g, device="cuda").bfloat16()
    logits = x.double() @ L.tensors["router_w"].double()
    if L.tensors["router_bias"] is not None:
        logits = logits + L.tensors["router_bias"].double()
    idx, w, place, offsets = C.route_rows(logits, k)
    z = C.shared_proj(shape, x, L.tensors["U_gate"], L.tensors["U_up"])
    y = C.vq_lr_expert_ffn(shape, x, idx, w, z, L)
    assert torch.equal(y, C.vq_lr_expert_ffn(shape, x, idx.clone(), w.clone(), z, L))
    want, i, _ = C.moe_layer(shape, x, L)
    assert torch.equal(i, idx) and ((y - want).abs() <= 1e-5 * want.abs().max()).all()


def test_outputs_are_apart(C):
    z = torch.randn((5, 16), generator=torch.Generator().manual_seed(1)).cuda()
    idx, w, place, offsets = C.route_rows(z, 3)
    parts = [idx, w, place, offsets]
    assert all(t.data_ptr() % 16 == 0 for t in parts)
    assert len({t.untyped_storage().data_ptr() for t in parts}) == 4
    x = torch.ones((5, 3), device="cuda", requires_grad=True)
    kept = w.clone()
    loss = (x * w).sum()            # keeps the weights for its gradient
    idx.clamp_(min=0)
    place.add_(1)
    loss.backward()
    assert torch.equal(x.grad, kept) and torch.equal(w, kept)
