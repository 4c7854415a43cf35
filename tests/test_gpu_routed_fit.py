"""The router, the rows to their experts and back, the feed-forward block and the
optimizer together, as a training step of a routed layer runs them.

Bounds of the factors' gradients: those of tests/test_gpu_distill_fit.py (3
percent in the 2-norm, the roundings to bf16 on the way). The router's gradient
is a difference of the weights' gradients, each with these roundings and the
experts' outputs' own: sqrt(2) times 3 percent, 4.5 percent is the bound.
"""

import numpy as np
import pytest
import torch
from test_gpu_distill_fit import _setup

from paper_2609_21137_amd import fit

pytestmark = pytest.mark.gpu

F64 = torch.float64


@pytest.fixture(scope="module")
def C():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_21137_amd import cardan
    return cardan


def _weights(z, idx, routing):
    s = torch.sigmoid(z) if routing.get("score") == "sigmoid" else torch.softmax(z, 1)
    w = s.gather(1, idx)
    if routing.get("renorm", True):
        w = w / w.sum(1, keepdim=True)
    return w * routing.get("scale", 1.0)


def _plain(student, x, head, teacher, ids, labels, T, c):
    """The step in float64 at the experts that the layer chose; (loss, gradients)."""
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
    rw = F.get("router_w", student.router_w.double())
    rb = F.get("router_bias", None if student.router_bias is None else student.router_bias.double())
    z = X @ rw + (0 if rb is None else rb)
    idx = student.route(x)[0]
    a = _weights(z, idx, student.routing)
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
    return {n: t.grad for n, t in F.items()}


ROUTINGS = [{}, dict(score="sigmoid", scale=2.0), dict(renorm=False), dict(score="sigmoid", groups=3, top_groups=2, group_best=2)]


@pytest.mark.parametrize("act", ["silu_glu", "relu2_up"])
@pytest.mark.parametrize("which", range(len(ROUTINGS)))
@pytest.mark.parametrize("router", [False, True])
def test_gradients_of_a_step(C, act, which, router):
    L, k, d, x, head, teacher, ids, labels = _setup(act, 8, False)
    routing = dict(ROUTINGS[which])
    if which == 1:
        routing["bias"] = torch.linspace(-0.2, 0.2, 6, device="cuda")
    student = fit.TrainedLayer(L, k, d, act, routing=routing, train_router=router)
    want = _plain(student, x, head, teacher, ids, labels, 2.0, 0.5)
    loss, got = fit.distill_step(student, x, head, teacher, ids, labels=labels, temperature=2.0, ce_weight=0.5)
    assert set(got) == set(want) == set(student.factors) and router == ("router_w" in got)
    for n in want:
        rel = float((got[n].double() - want[n]).norm() / want[n].norm())
        assert rel <= (0.045 if n.startswith("router") else 0.03), f"{n}: {rel:.3e}"
    again = fit.distill_step(student, x, head, teacher, ids, labels=labels, temperature=2.0, ce_weight=0.5)[1]
    assert all(torch.equal(got[n], again[n]) for n in got)


def test_default_routing_is_the_layers(C):
    """With routing={} the selection and the weights are those of the softmax over the kept logits,
    and the sums of the same bf16 rows in float32 differ by their order alone (k 2^-24 of the sizes)."""
    L, k, d, x, *_ = _setup("silu_glu", 8, False)
    a, b = fit.TrainedLayer(L, k, d), fit.TrainedLayer(L, k, d, routing={})
    (i, w), (j, v) = a.route(x), b.route(x)
    assert torch.equal(i, j) and ((w - v).abs() <= 2.0 ** -23 * w).all()
    ya, yb = a.forward(x), b.forward(x)
    ye = a._kept[5]
    assert ((ya - yb).abs() <= 1e-5 * ya.abs().max()).all() and ye is not None


@pytest.mark.parametrize("optimizer", ["adamw", "adamw8"])
@pytest.mark.parametrize("router", [False, True])
def test_distilled_layer_runs(C, optimizer, router):
    L, k, d, x, head, teacher, ids, labels = _setup("silu_glu", 8, False)
    out, history = fit.distill_layer(L, x, head, teacher, ids, k, d, labels=labels, temperature=2.0, ce_weight=0.5, steps=3,
                                     rows=40, lr=1e-3, optimizer=optimizer, weight_decay=0.01, train_router=router)
    assert history.shape == (3, 2) and np.isfinite(history).all()
    assert out["U_gate"] is out["U_up"]
    assert router == (out["router_w"] is not L["router_w"])
    if router:
        assert out["router_w"].dtype == L["router_w"].dtype and out["router_bias"].dtype == np.float32
        assert not np.array_equal(out["router_w"], L["router_w"])
    shape = C.make_shape(128, 64, 6, k, d, 16, 8)
    y, idx, w = C.moe_layer(shape, x[:8].contiguous(), C.DeviceLayer.from_numpy(out))
    student = fit.TrainedLayer(out, k, d)
    torch.cuda.synchronize()
    assert torch.isfinite(y).all() and torch.equal(idx.long(), student.route(x[:8])[0])


def test_adamw_without_decay_takes_adams_steps(C):
    """The same batches: weights are off by the steps' roundings, 20 2^-24 of 3 lr and 3 2^-24 of themselves a
    step, and what the gradients make of that (an update's sign, where a gradient is near zero, is left out by the
    median)."""
    L, k, d, x, head, teacher, ids, labels = _setup("silu_glu", 8, False)
    args = dict(labels=labels, temperature=2.0, ce_weight=0.5, steps=3, rows=40, lr=1e-3)
    a, _ = fit.distill_layer(L, x, head, teacher, ids, k, d, **args)
    b, _ = fit.distill_layer(L, x, head, teacher, ids, k, d, optimizer="adamw", **args)
    for n in ("cb_up", "V_up", "A_down", "B_down"):
        diff = np.abs(fit.bf16_value(a[n]) - fit.bf16_value(b[n]))
        assert np.median(diff) == 0.0 and diff.max() <= 6e-3


def test_refusals(C):
    L, k, d, x, head, teacher, ids, labels = _setup("silu_glu", 8, False)
    with pytest.raises(ValueError):
        fit.distill_layer(L, x, head, teacher, ids, k, d, optimizer="sgd")
    with pytest.raises(ValueError):
        fit.distill_layer(L, x, head, teacher, ids, k, d, weight_decay=0.1)
    with pytest.raises(ValueError):
        fit.TrainedLayer(L, k, d, routing=dict(score="tanh")).forward(x)


def test_a_batch_without_rows(C):
    L, k, d, x, head, teacher, ids, labels = _setup("silu_glu", 8, False)
    student = fit.TrainedLayer(L, k, d, routing={}, train_router=True)
    loss, grads = fit.distill_step(student, x[:0], head, teacher[:0], ids[:0], labels=labels[:0])
    assert loss.shape == (0, 2) and set(grads) == set(student.factors)
    assert all((g == 0).all() and g.shape == student.factors[n].shape for n, g in grads.items())


@pytest.mark.parametrize("N,pad", [(1, 0), (50, 7), (300, 40)])
def test_all_operators_in_turn(C, N, pad):
    """Routing with a padded end, rows to the experts, the block, rows back, every gradient and an
    AdamW step of float32 weights with their bf16 copies, against float64 at the same selection.
    Bounds: bf16 roundings of xe's products (h, ye), of dye, dg and du and of the results, 2^-8 each,
    six of them one after another: 6 2^-8 in the 2-norm if none cancelled; 3 percent."""
    H, I, E, k = 128, 64, 8, 3
    g = torch.Generator(device="cuda").manual_seed(N)

    def draw(*shape, std=1.0):
        return torch.randn(shape, generator=g, device="cuda") * std

    x = draw(N, H).bfloat16()
    logits = draw(N, E, std=2.0)
    logits[N - pad:] = -float("inf")
    master = [draw(E, H, I, std=H ** -0.5), draw(E, H, I, std=H ** -0.5), draw(E, I, H, std=I ** -0.5)]
    W = [m.bfloat16() for m in master]
    master = [w.float() for w in W]
    dy = draw(N, H).bfloat16()
    o = dict(score="sigmoid", scale=2.5, groups=4, top_groups=2, group_best=2)
    bias = draw(E, std=0.1)
    idx, a, place, offsets = C.route_rows(logits, k, bias=bias, **o)
    xe = C.dispatch_rows(x, place)
    ye, saved = C.ffn_forward(xe, *W, offsets=offsets, save=True)
    y = C.combine_rows(ye, place, a)
    dye, da = C.combine_rows_backward(dy, ye, place, a)
    dxe, *dW = C.ffn_backward(dye, xe, *W, saved, offsets=offsets)
    dx = C.combine_rows(dxe, place)
    dz = C.route_rows_backward(logits, idx, da, **o)
    states = [C.adamw_state(m, 8) for m in master]
    before = [m.clone() for m in master]
    C.adamw_step(master, dW, states, 1, 1e-3, weight_decay=0.1, copies=W)
    torch.cuda.synchronize()

    live = N - pad
    assert (idx[live:] == -1).all() and (place[live:] == -1).all() and (y[live:] == 0).all() and (dx[live:] == 0).all()
    assert (dz[live:] == 0).all() and (da[live:] == 0).all()
    assert int(offsets[-1]) == live * k
    X = x[:live].double().requires_grad_(True)
    Z = logits[:live].double().requires_grad_(True)
    Ws = [m.double().requires_grad_(True) for m in before]
    s = torch.sigmoid(Z).gather(1, idx[:live].long())
    w = s / s.sum(1, keepdim=True) * 2.5
    Y = torch.zeros((live, H), dtype=F64, device="cuda")
    for e in range(E):
        we = (w * (idx[:live] == e)).sum(1, keepdim=True)
        Y = Y + we * ((torch.nn.functional.silu(X @ Ws[0][e]) * (X @ Ws[1][e])) @ Ws[2][e])
    (Y * dy[:live].double()).sum().backward()
    for got, want, name in ((y[:live], Y.detach(), "y"), (dx[:live], X.grad, "dx"), (dz[:live], Z.grad, "dz"),
                            *((q, t.grad, n) for q, t, n in zip(dW, Ws, ("gate", "up", "down")))):
        rel = float((got.double() - want).norm() / want.norm())
        assert rel <= (0.045 if name == "dz" else 0.03), f"{name}: {rel:.3e}"
    for m, b, q, c in zip(master, before, dW, W):
        # the first step: m / (1 - b1) over the root of v / (1 - b2) is the gradient over its size
        q = q.double()
        want = b.double() * (1 - 1e-4) - 1e-3 * q / (q.abs() + 1e-8)
        assert ((m.double() - want).abs() <= 1e-3 * 20 * 2.0 ** -24 + 4 * 2.0 ** -24 * b.double().abs()).all()
        assert torch.equal(c, m.bfloat16())
