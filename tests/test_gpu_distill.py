"""The distillation loss and its gradient against the formulas in float64.

Bounds, per row. Losses: a probability's logarithm is a difference of the
logit to the row's log-sum; the sum of V float32 exponentials, each within 2^-20
of its value, and their adding, at most V roundings of 2^-24 but spread over the
threads' partial sums, stay below 2^-19 relative, so a logarithm is off by
2^-19 plus 2^-22 of its size. Gradients: each exponential within 2^-19 (1 + |s -
lse| / T 2^-3) of its value, the differences of two terms rounded in float32,
and the output's own rounding (half a step).
"""

import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

E19 = 2.0 ** -19


@pytest.fixture(scope="module")
def C():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_21137_amd import cardan
    return cardan


def _say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def _inputs(N, V, K, dtype, seed, pad=0, offset=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    full = (torch.randn((N, V + pad + offset), generator=g, device="cuda") * 2).to(dtype)
    logits = full[:, offset:offset + V]
    ids = torch.stack([torch.randperm(V, generator=g, device="cuda")[:K] for _ in range(N)]).int()
    teacher = torch.sort(torch.randn((N, K), generator=g, device="cuda") * 3, dim=1, descending=True).values.contiguous()
    labels = torch.randint(0, V, (N,), generator=g, device="cuda").int()
    weight = torch.randn((N,), generator=g, device="cuda")
    return logits, teacher, ids, labels, weight


def _oracle(logits, teacher, ids, labels, T, c, w):
    z, t = logits.double(), teacher.double()
    N, V = z.shape
    ok = (ids >= 0) & (ids < V)
    tp = torch.where(ok, t / T, -torch.inf)
    some = ok.any(1)
    p = torch.where(some[:, None], torch.softmax(torch.where(some[:, None], tp, 0.0), 1), 0.0)
    p = torch.where(ok, p, 0.0)
    lq, l1 = torch.log_softmax(z / T, 1), torch.log_softmax(z, 1)
    at = ids.clamp(0, V - 1).long()
    term = torch.where(p > 0, p * (torch.log(p.clamp(min=1e-300)) - lq.gather(1, at)), 0.0)
    size = torch.where(p > 0, p * (torch.log(p.clamp(min=1e-300)).abs() + lq.gather(1, at).abs()), 0.0)
    kd = T * T * term.sum(1)
    lab = (labels >= 0) & (labels < V) if labels is not None else torch.zeros(N, dtype=torch.bool, device=z.device)
    la = labels.clamp(0, V - 1).long() if labels is not None else torch.zeros(N, dtype=torch.long, device=z.device)
    ce = torch.where(lab, -l1.gather(1, la[:, None])[:, 0], 0.0)
    loss = torch.stack([torch.where(some, kd, 0.0), ce], 1)
    eloss = torch.stack([T * T * (2 * E19 + E19 * size.sum(1)), 2 * E19 + E19 * ce.abs()], 1)
    wd = w.double() if w is not None else torch.ones(N, dtype=torch.float64, device=z.device)
    a, b = wd * T * some, wd * c * lab
    tgt = torch.zeros_like(z).scatter_add_(1, at, p)
    hot = torch.zeros_like(z).scatter_(1, la[:, None], 1.0)
    q, r = torch.exp(lq), torch.exp(l1)
    grad = a[:, None] * (q - tgt) + b[:, None] * (r - hot)
    egrad = E19 * (a.abs()[:, None] * (q * (1 + lq.abs() / 8) + tgt) + b.abs()[:, None] * (r * (1 + l1.abs() / 8) + hot))
    return loss, eloss, grad, egrad


def _check(got, dlogits, want, dtype):
    loss, eloss, grad, egrad = want
    d = (got.double() - loss).abs()
    assert (d <= eloss).all(), f"loss off by {float((d - eloss).max()):.2e} past its bound"
    if dlogits is not None:
        half = torch.finfo(dtype).eps / 2
        d = (dlogits.double() - grad).abs()
        tol = half * 1.01 * grad.abs() + 1.01 * egrad + 1e-37
        bad = d > tol
        assert not bad.any(), f"{int(bad.sum())} gradients past their bound, first at {bad.nonzero()[0].tolist()}"


CASES = [
    # N, V, K, type, T, ce, pad, offset
    (1, 1, 1, torch.bfloat16, 1.0, 1.0, 0, 0),
    (1, 7, 3, torch.float32, 2.0, 0.5, 0, 0),
    (2, 8, 8, torch.bfloat16, 0.5, 0.0, 0, 0),
    (3, 129, 5, torch.bfloat16, 2.0, 0.5, 0, 0),
    (5, 1001, 64, torch.float32, 1.0, 0.25, 3, 0),
    (17, 4097, 256, torch.bfloat16, 3.0, 1.0, 0, 0),
    (4, 5000, 1, torch.bfloat16, 2.0, 0.5, 8, 0),
    (6, 33003, 1024, torch.bfloat16, 2.0, 0.5, 5, 8),
    (1, 32000, 256, torch.bfloat16, 1.0, 0.0, 0, 0),
    (9, 50257, 256, torch.bfloat16, 2.0, 0.5, 0, 0),
    (3, 128256, 100, torch.float32, 4.0, 2.0, 64, 0),
    (300, 2050, 32, torch.bfloat16, 1.5, 0.5, 0, 0),
    (2, 262144, 256, torch.bfloat16, 2.0, 0.5, 0, 0),
    (2, 400001, 17, torch.float32, 2.0, 0.5, 0, 0),
]


@pytest.mark.parametrize("N,V,K,dtype,T,c,pad,offset", CASES)
def test_loss_and_gradient(C, N, V, K, dtype, T, c, pad, offset):
    _say(f"[distill] N={N} V={V} K={K} {dtype} T={T} c={c} pad={pad}")
    logits, teacher, ids, labels, w = _inputs(N, V, K, dtype, seed=V, pad=pad, offset=offset)
    want = _oracle(logits, teacher, ids, labels, T, c, w)
    loss, d = C.distill_loss(logits, teacher, ids, labels=labels, temperature=T, ce_weight=c, row_weight=w)
    _check(loss, d, want, dtype)
    # the loss alone, the gradient in place of the logits, and without labels or weights
    alone, none = C.distill_loss(logits, teacher, ids, labels=labels, temperature=T, ce_weight=c, row_weight=w,
                                 grad=False)
    assert none is None
    _check(alone, None, want, dtype)
    bare = _oracle(logits, teacher, ids, None, T, c, None)
    l2, d2 = C.distill_loss(logits, teacher, ids, temperature=T, ce_weight=c)
    _check(l2, d2, bare, dtype)
    whole = logits._base if logits._base is not None else logits
    keep = whole.clone()
    l3, d3 = C.distill_loss(logits, teacher, ids, labels=labels, temperature=T, ce_weight=c, row_weight=w,
                            dlogits=logits)
    assert d3.data_ptr() == logits.data_ptr() and torch.equal(l3, loss) and torch.equal(d3, d)
    outside = torch.ones_like(whole, dtype=torch.bool)
    outside[:, offset:offset + V] = False
    assert torch.equal(whole[outside], keep[outside])


def test_rows_without_entries_or_labels(C):
    N, V, K = 12, 3001, 40
    for dtype in (torch.bfloat16, torch.float32):
        logits, teacher, ids, labels, w = _inputs(N, V, K, dtype, seed=7)
        ids[0], labels[0] = -1, -100                  # nothing: zero loss and gradient
        ids[1] = -1                                   # a label alone
        labels[2] = -1                                # a teacher alone
        ids[3, 5:] = -1                               # few entries
        ids[4, 3] = V                                 # outside the vocabulary: absent
        labels[5] = V + 3
        ids[6] = 2 ** 31 - 1
        labels[6] = -2 ** 31
        logits[0, 7] = float("nan")                   # not looked at
        teacher[3, 5:] = float("nan")                 # absent entries' values are not looked at
        teacher[4, 3] = float("inf")
        clean = logits.clone()
        clean[0] = 0.0
        tc = torch.nan_to_num(teacher, 0.0, 0.0, 0.0)
        want = _oracle(clean, tc, ids, labels, 2.0, 0.5, w)
        loss, d = C.distill_loss(logits, teacher, ids, labels=labels, temperature=2.0, ce_weight=0.5, row_weight=w)
        _check(loss, d, want, dtype)
        for n in (0, 6):
            assert (loss[n] == 0).all() and (d[n] == 0).all()


def test_entries_named_twice(C):
    """An entry named several times counts with all its probabilities, also where it is the label."""
    N, V, K = 6, 900, 33
    logits, teacher, ids, labels, w = _inputs(N, V, K, torch.float32, seed=11)
    ids[0] = 5
    ids[1, ::2] = 17
    labels[1] = 17
    ids[2, 3] = ids[2, 30]
    ids[3, :] = torch.arange(K, device="cuda") % 4
    labels[3] = 2
    want = _oracle(logits, teacher, ids, labels, 2.0, 0.5, w)
    out = [C.distill_loss(logits, teacher, ids, labels=labels, temperature=2.0, ce_weight=0.5, row_weight=w)
           for _ in range(3)]
    for loss, d in out:
        _check(loss, d, want, torch.float32)
        assert torch.equal(d, out[0][1]) and torch.equal(loss, out[0][0])


def test_masked_and_extreme_logits(C):
    N, V, K = 8, 5003, 24
    for dtype in (torch.bfloat16, torch.float32):
        logits, teacher, ids, labels, w = _inputs(N, V, K, dtype, seed=13)
        low = torch.finfo(dtype).min
        free = torch.ones((N, V), dtype=torch.bool, device="cuda").scatter_(1, ids.long(), False)
        free.scatter_(1, labels.long()[:, None], False)
        logits[0].masked_fill_(free[0], float("-inf"))  # everything else masked out
        logits[1].masked_fill_(free[1], low)
        logits[2] = low                                 # a row of the lowest value: uniform
        logits[3] *= 50.0                               # far apart
        logits[4, ids[4, 0].long()] = 30000.0           # one that is everything
        teacher[5] = torch.finfo(torch.float32).min     # uniform over its entries
        teacher[6, 1:] = float("-inf")                  # a single entry
        want = _oracle(logits, teacher, ids, labels, 2.0, 0.5, w)
        loss, d = C.distill_loss(logits, teacher, ids, labels=labels, temperature=2.0, ce_weight=0.5, row_weight=w)
        assert torch.isfinite(d).all()
        _check(loss, d, want, dtype)
        logits[0, 1] = float("nan")
        logits[1, 2] = float("inf")
        loss2, d2 = C.distill_loss(logits, teacher, ids, labels=labels, temperature=2.0, ce_weight=0.5, row_weight=w)
        assert torch.isnan(loss2[0]).all() and torch.isnan(d2[:2]).any(1).all()
        assert torch.equal(loss2[2:], loss[2:]) and torch.equal(d2[2:], d[2:])


@pytest.mark.parametrize("T", [1.0, 2.0, 3.0])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_teacher_rows_masked_out(C, dtype, T):
    N, V, K = 7, 1003, 70
    logits, teacher, ids, labels, w = _inputs(N, V, K, dtype, 31)
    low = float("-inf")
    teacher[0] = low                        # nothing left, with a label
    teacher[1] = low                        # nothing left, nothing else
    labels[1] = -1
    teacher[2, ::2] = low                   # a part, the label at a masked entry
    labels[2] = ids[2, 4]
    teacher[3, 1:] = low                    # the label at a masked entry of a row with one left
    labels[3] = ids[3, 9]
    teacher[4] = low                        # nothing left, the label at a masked entry
    labels[4] = ids[4, 0]
    teacher[5, 3] = float("nan")
    teacher[6, 3] = float("inf")
    _say(f"teacher rows masked out: {dtype} T={T}")
    loss, d = C.distill_loss(logits, teacher, ids, labels, T, 0.5, w)
    n = 5
    seen = torch.where(teacher == low, -1, ids)[:n].contiguous()
    want = _oracle(logits[:n], torch.where(teacher == low, 0.0, teacher)[:n], seen, labels[:n], T, 0.5, w[:n])
    _check(loss[:n], d[:n], want, dtype)
    assert (loss[[0, 1, 4], 0] == 0).all() and (d[1] == 0).all() and loss[1, 1] == 0
    for i in (5, 6):
        assert torch.isnan(loss[i, 0]) and torch.isnan(d[i, ids[i].long()]).all() and torch.isfinite(loss[i, 1])


def test_gradient_against_differences(C):
    N, V, K, T, c = 4, 777, 20, 2.0, 0.5
    logits, teacher, ids, labels, w = _inputs(N, V, K, torch.float32, seed=3)
    _, d = C.distill_loss(logits, teacher, ids, labels=labels, temperature=T, ce_weight=c, row_weight=w)

    def f(z):
        loss = _oracle(z, teacher, ids, labels, T, c, w)[0]
        return float((w.double() * (loss[:, 0] + c * loss[:, 1])).sum())

    g = torch.Generator(device="cuda").manual_seed(1)
    for _ in range(4):
        v = torch.randn((N, V), generator=g, device="cuda", dtype=torch.float64)
        want = (f(logits.double() + 1e-5 * v) - f(logits.double() - 1e-5 * v)) / 2e-5
        # float32 gradients: 2^-18 of the terms' sizes at most; the differences' own error is 1e-9
        assert abs(float((d.double() * v).sum()) - want) <= 2.0 ** -18 * float((d.double() * v).abs().sum()) + 1e-8


def test_streams_and_graphs(C):
    for N, V in ((2, 9001), (400, 3000)):
        logits, teacher, ids, labels, w = _inputs(N, V, 50, torch.bfloat16, seed=V)
        call = lambda **k: C.distill_loss(logits, teacher, ids, labels=labels, temperature=2.0, ce_weight=0.5,  # noqa: E731
                                          row_weight=w, **k)
        loss, d = call()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            l2, d2 = call()
        side.synchronize()
        assert torch.equal(l2, loss) and torch.equal(d2, d)
        outs, graphs = [], []
        for _ in range(2):
            o, g = torch.empty_like(loss), torch.empty_like(d)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                call(out=o, dlogits=g)
            outs.append((o, g))
            graphs.append(graph)
        for _ in range(3):
            for graph, (o, g) in zip(graphs, outs):
                o.fill_(5.0)
                g.fill_(5.0)
                graph.replay()
            call()
            torch.cuda.synchronize()
            for o, g in outs:
                assert torch.equal(o, loss) and torch.equal(g, d)


def test_labels_alone_and_other_row_strides(C):
    """No teacher (K = 0) is the cross entropy; a gradient may have rows of its own alignment."""
    for V, dtype in ((4097, torch.bfloat16), (1003, torch.float32)):
        N = 7
        logits, teacher, ids, labels, w = _inputs(N, V, 5, dtype, seed=V)
        none_t, none_i = teacher[:, :0].contiguous(), ids[:, :0].contiguous()
        loss, d = C.distill_loss(logits, none_t, none_i, labels=labels, temperature=3.0, ce_weight=1.5, row_weight=w)
        gone = torch.full_like(ids, -1)
        want = _oracle(logits, teacher, gone, labels, 3.0, 1.5, w)
        _check(loss, d, want, dtype)
        assert (loss[:, 0] == 0).all()
        l0, d0 = C.distill_loss(logits, teacher, ids, labels=labels, temperature=3.0, ce_weight=1.5, row_weight=w)
        out = torch.full((N, V + 3), 7.0, dtype=dtype, device="cuda")
        l1, d1 = C.distill_loss(logits, teacher, ids, labels=labels, temperature=3.0, ce_weight=1.5, row_weight=w,
                                dlogits=out[:, :V])
        assert torch.equal(d1, d0) and torch.equal(l0, l1) and (out[:, V:] == 7.0).all()


def test_temperatures(C):
    """From a hard maximum to a flat one."""
    N, V, K = 5, 2111, 16
    logits, teacher, ids, labels, w = _inputs(N, V, K, torch.float32, seed=2)
    for T in (2.0 ** -6, 0.25, 2.0, 64.0):
        want = _oracle(logits, teacher, ids, labels, T, 0.5, w)
        loss, d = C.distill_loss(logits, teacher, ids, labels=labels, temperature=T, ce_weight=0.5, row_weight=w)
        loss_ref, eloss, grad, egrad = want
        # an exponent's own rounding grows with its size: |s - max| / T 2^-24, up to 24 / T here
        scale = max(1.0, 1.0 / T)
        _check(loss, d, (loss_ref, eloss * scale, grad, egrad * scale), torch.float32)


def test_refusals(C):
    logits, teacher, ids, labels, w = _inputs(3, 50, 4, torch.bfloat16, seed=1)
    with pytest.raises(ValueError):
        C.distill_loss(logits.t(), teacher, ids)
    with pytest.raises(ValueError):
        C.distill_loss(logits, teacher, ids.long())
    with pytest.raises(ValueError):
        C.distill_loss(logits, teacher.bfloat16(), ids)
    with pytest.raises(ValueError):
        C.distill_loss(logits, teacher, ids[:, :3])
    with pytest.raises(ValueError):
        C.distill_loss(logits, teacher, ids, labels=labels.cpu())
    with pytest.raises(ValueError):
        C.distill_loss(logits.expand(3, 50)[:1].expand(3, 50), teacher, ids)
    with pytest.raises(C.CardanError):
        C.distill_loss(logits, teacher, ids, temperature=0.0)


def test_no_rows(C):
    e = torch.empty((0, 100), dtype=torch.bfloat16, device="cuda")
    t = torch.empty((0, 4), device="cuda")
    loss, d = C.distill_loss(e, t, t.int())
    assert loss.shape == (0, 2) and d.shape == (0, 100)
