"""The training calls of the binding leave autograd alone: outputs carry no graph."""

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_outputs_carry_no_graph():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_21137_amd import cardan as C
    bf = torch.bfloat16
    x = torch.randn((5, 128), device="cuda").to(bf).requires_grad_(True)
    W = [(torch.randn(s, device="cuda") * 0.1).to(bf).requires_grad_(True) for s in ((128, 64), (128, 64), (64, 128))]
    y, saved = C.ffn_forward(x, *W, save=True)
    grads = C.ffn_backward(torch.ones_like(y), x, *W, saved)
    logits = torch.randn((5, 50), device="cuda", requires_grad=True)
    loss, d = C.distill_loss(logits, torch.zeros((5, 2), device="cuda"), torch.ones((5, 2), device="cuda").int())
    for t in (y, *saved, *grads, loss, d):
        assert not t.requires_grad and t.grad_fn is None
    assert all(t.grad is None for t in (x, *W, logits))
