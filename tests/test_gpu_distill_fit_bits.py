"""How many bits the distillation step's gradients keep on their way."""

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


@pytest.mark.parametrize("act", ["silu_glu", "relu2_up"])
def test_gradient_behind_the_head_is_float32(C, act, monkeypatch):
    """The layer's upstream gradient is the float32 product of the logits' gradient with
    the head: a sum of V products of bf16 values (exact in float32), off by at most
    (V + 2) 2^-24 of the sum of their sizes."""
    L, k, d, x, head, teacher, ids, labels = _setup(act, 8, False)
    student = fit.TrainedLayer(L, k, d, act)
    seen = {}
    whole, back = C.distill_loss, student.backward

    def loss(*a, **kw):
        out = whole(*a, **kw)
        seen["dlogits"] = out[1].clone()
        return out

    def backward(dy):
        seen["dy"] = dy.clone()
        return back(dy)

    monkeypatch.setattr(C, "distill_loss", loss)
    monkeypatch.setattr(student, "backward", backward)
    fit.distill_step(student, x, head, teacher, ids, labels=labels, temperature=2.0, ce_weight=0.5)
    g, h = seen["dlogits"].double(), head.double().t().contiguous()
    assert seen["dy"].dtype == torch.float32
    err = (seen["dy"].double() - g @ h).abs()
    assert (err <= (head.shape[1] + 2) * 2.0 ** -24 * (g.abs() @ h.abs())).all()


@pytest.mark.parametrize("act", ["silu_glu", "relu2_up"])
def test_a_batch_without_rows(C, act):
    L, k, d, x, head, teacher, ids, labels = _setup(act, 8, False)
    student = fit.TrainedLayer(L, k, d, act)
    loss, grads = fit.distill_step(student, x[:0], head, teacher[:0], ids[:0], labels=labels[:0])
    assert loss.shape == (0, 2) and set(grads) == set(student.factors)
    assert all((g == 0).all() and g.shape == student.factors[n].shape for n, g in grads.items())
