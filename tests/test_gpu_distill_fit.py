"""The distillation stage of the offline fit: the feed-forward block, its
gradients and the distillation loss together, as ``fit`` uses them.

The gradients are compared with torch's float64 differentiation of the whole
step written out plainly (decode, low-rank terms, routing, experts, head,
loss). Their bound counts the roundings to bf16 that the step makes on the way:
the expert matrices, h, each expert's output, the layer's output, the logits
(whose rounding, not relative to the differences that the loss sees, reaches a
probability as an exponent's error), their gradient, the rows' upstream
gradients, dg and du, and the weights' gradients. Each is off by at most
2^-8 of its value; ten of them, independent and of comparable weight, give 4
percent if all were largest and 1.3 percent as a root of squares; the logits'
rounding is up to 2^-8 times their size (about 4) in an exponent, as large
again as all others. 3 percent in the 2-norm is the bound.
"""

import sys

import numpy as np
import pytest
import torch

from paper_2609_21137_amd import fit, synth

pytestmark = pytest.mark.gpu


def _say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


@pytest.fixture(scope="module")
def C():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_21137_amd import cardan
    return cardan


def _setup(act, r, separate, N=96, V=1000, K=48):
    H, I, E, k, d = 128, 64, 6, 2, 4
    L = synth.make_layer(H, I, E, d, 16, r, 5)
    if act == "silu_glu" and separate and r:
        L["U_gate"] = L["U_up"].copy()
    # larger code words than the workloads': every term of the layer counts
    for n in ("cb_gate", "cb_up", "cb_down"):
        L[n] = synth.to_bf16_bits(fit.bf16_value(L[n]) * 4.0)
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((N, H), generator=g, device="cuda").bfloat16()
    head = (torch.randn((H, V), generator=g, device="cuda") * 0.5).bfloat16()
    ids = torch.stack([torch.randperm(V, generator=g, device="cuda")[:K] for _ in range(N)]).int()
    teacher = torch.randn((N, K), generator=g, device="cuda") * 2
    labels = torch.randint(0, V, (N,), generator=g, device="cuda").int()
    labels[::7] = -1
    return L, k, d, x, head, teacher, ids, labels


def _plain(student, x, head, teacher, ids, labels, T, c):
    """The step in float64 with autograd; returns (loss [N, 2], gradients)."""
    F = {n: t.double().requires_grad_(True) for n, t in student.factors.items()}
    W = {}
    for p in student._projections() + ["down"]:
        J = student.codes[p]
        E, nb, n_out = J.shape
        W[p] = F["cb_" + p][J].permute(0, 1, 3, 2).reshape(E, nb * student.d, n_out)
        left, right = student._lowrank(p)
        if left in F:
            W[p] = W[p] + torch.matmul(F[left], F[right])
    X = x.double()
    logits = X @ student.router_w.double() + (0 if student.router_bias is None else student.router_bias.double())
    val, idx = torch.topk(logits, student.k, dim=1)
    a = torch.softmax(val, 1)
    y = torch.zeros_like(X)
    for e in range(W["up"].shape[0]):
        w = (a * (idx == e)).sum(1, keepdim=True)
        u = X @ W["up"][e]
        h = torch.nn.functional.silu(X @ W["gate"][e]) * u if student.gated else torch.relu(u) ** 2
        y = y + w * (h @ W["down"][e])
    z = y @ head.double()
    tp = torch.softmax(teacher.double() / T, 1)
    lq = torch.log_softmax(z / T, 1).gather(1, ids.long())
    kd = T * T * (tp * (tp.log() - lq)).sum(1)
    on = labels >= 0
    ce = -torch.log_softmax(z, 1).gather(1, labels.clamp(min=0).long()[:, None])[:, 0] * on
    (kd + c * ce).mean().backward()
    return torch.stack([kd, ce], 1).detach(), {n: t.grad for n, t in F.items()}


@pytest.mark.parametrize("act,r,separate", [("silu_glu", 8, False), ("silu_glu", 8, True), ("silu_glu", 0, False),
                                            ("relu2_up", 8, False)])
def test_gradients_of_a_step(C, act, r, separate):
    _say(f"[distill fit] {act} r={r} separate={separate}")
    L, k, d, x, head, teacher, ids, labels = _setup(act, r, separate)
    student = fit.TrainedLayer(L, k, d, act)
    want_loss, want = _plain(student, x, head, teacher, ids, labels, 2.0, 0.5)
    loss, got = fit.distill_step(student, x, head, teacher, ids, labels=labels, temperature=2.0, ce_weight=0.5)
    assert set(got) == set(want) == set(student.factors)
    assert (r == 0) == ("V_up" not in got) and ("U_gate" in got) == (separate and act == "silu_glu" and r > 0)
    # a loss is a difference of logits (and a mean of them): 2^-8 of their sizes, twice, plus the layer's roundings
    size = float((student.forward(x).bfloat16() @ head).abs().max())
    assert (loss.double() - want_loss).abs().max() <= 4.0 * 4 * 2.0 ** -8 * size
    for n in want:
        rel = float((got[n].double() - want[n]).norm() / want[n].norm())
        assert rel <= 0.03, f"{n}: {rel:.3e}"
    again = fit.distill_step(student, x, head, teacher, ids, labels=labels, temperature=2.0, ce_weight=0.5)[1]
    assert all(torch.equal(got[n], again[n]) for n in got)


def test_distilled_layer_runs(C):
    """Adam steps return a layer in storage formats that the layer call takes,
    whose codes and router are the fitted ones."""
    L, k, d, x, head, teacher, ids, labels = _setup("silu_glu", 8, False)
    out, history = fit.distill_layer(L, x, head, teacher, ids, k, d, labels=labels, temperature=2.0, ce_weight=0.5,
                                     steps=3, rows=40, lr=1e-3)
    assert history.shape == (3, 2) and np.isfinite(history).all()
    assert out["U_gate"] is out["U_up"]
    for n in ("codes_gate", "codes_up", "codes_down", "router_w"):
        assert out[n] is L[n]
    assert any(not np.array_equal(out[n], L[n]) for n in ("cb_up", "V_up", "A_down"))
    shape = C.make_shape(128, 64, 6, k, d, 16, 8)
    y, idx, w = C.moe_layer(shape, x[:8].contiguous(), C.DeviceLayer.from_numpy(out))
    student = fit.TrainedLayer(out, k, d)
    want = student.forward(x[:8].contiguous())
    torch.cuda.synchronize()
    assert torch.isfinite(y).all()
    assert torch.equal(idx.long(), student.route(x[:8])[0])
    # the student's experts are bf16 matrices and its hidden rows and outputs bf16: three roundings
    assert float((y - want).norm() / want.norm()) <= 3 * 2.0 ** -8


def test_no_forward_no_backward(C):
    L, k, d, x, *_ = _setup("silu_glu", 0, False)
    with pytest.raises(RuntimeError):
        fit.TrainedLayer(L, k, d).backward(torch.zeros((4, 128), device="cuda"))
    with pytest.raises(ValueError):
        fit.TrainedLayer(L, k, d, act="gelu")
