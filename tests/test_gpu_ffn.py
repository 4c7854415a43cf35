"""The feed-forward block, forward and backward, against its formulas in float64.

Two bounds hold at once. Element by element: the roundings' worst case, carried
through the formulas (a sum of n products in float32 is off by at most (n + 2)
2^-24 of the sum of the products' sizes, bf16 rounds by at most 2^-8 of the
value, the activation in float32 by at most 2^-18 of its terms). In the 2-norm:
each rounding to bf16 is uniform within half a step, 2^-8 / sqrt(3) of the value
at most, and the roundings are independent, so two of them (the value that
enters the last product, and the output) give sqrt(2) of that; 10 % is added for
the rounding errors' own scatter on small outputs. The second bound is the
sharper one: one missing product of a sum of n changes it by 1 / sqrt(n).
"""

import math
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

B8, F24, ACT = 2.0 ** -8, 2.0 ** -24, 2.0 ** -18


@pytest.fixture(scope="module")
def C():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_21137_amd import cardan
    return cardan


def _say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def _inputs(N, E, H, I, act, seed, counts=None, first=0):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def n(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(torch.bfloat16)

    x, dy = n(N, H), n(N, H, std=0.1)
    Wg = n(E, H, I, std=H ** -0.5) if act == "silu_glu" else None
    Wu, Wd = n(E, H, I, std=H ** -0.5), n(E, I, H, std=I ** -0.5)
    off = None
    if counts is not None:
        off = torch.tensor([first] + [first + sum(counts[:i + 1]) for i in range(E)], dtype=torch.int32, device="cuda")
    return x, dy, Wg, Wu, Wd, off


def _gam(n):
    return (n + 2) * F24


def _oracle(x, dy, Wg, Wu, Wd, rows):
    """Values and worst-case errors of every output, in float64. ``rows``: [(lo, hi)] per group."""
    E, H, I = Wu.shape
    D = lambda t: t.double()  # noqa: E731
    val = {"y": torch.zeros_like(D(x)), "dx": torch.zeros_like(D(x)), "dWu": torch.zeros_like(D(Wu)),
           "dWd": torch.zeros_like(D(Wd))}
    if Wg is not None:
        val["dWg"] = torch.zeros_like(D(Wu))
    err = {k: torch.zeros_like(v) for k, v in val.items()}
    for e, (lo, hi) in enumerate(rows):
        if hi <= lo:
            continue
        X, Y, U, Dn = D(x[lo:hi]), D(dy[lo:hi]), D(Wu[e]), D(Wd[e])
        n = hi - lo
        u = X @ U
        eu = _gam(H) * (X.abs() @ U.abs())
        dh = Y @ Dn.T.contiguous()
        edh = _gam(H) * (Y.abs() @ Dn.T.contiguous().abs())
        if Wg is not None:
            G = D(Wg[e])
            g = X @ G
            eg = _gam(H) * (X.abs() @ G.abs())
            s = torch.sigmoid(g)
            ds = s + g * s * (1 - s)                                  # silu'
            dds = s * (1 - s) * (2 + g * (1 - 2 * s))                 # silu''
            h = g * s * u
            eh = (ds * u).abs() * eg + (g * s).abs() * eu + (B8 + ACT) * h.abs()
            dg, du = dh * u * ds, dh * g * s
            edg = ((u * ds).abs() * edh + (dh * ds).abs() * eu + (dh * u * dds).abs() * eg + B8 * dg.abs()
                   + ACT * (dh * u).abs() * (1 + g.abs() * s))
            edu = (g * s).abs() * edh + (dh * ds).abs() * eg + (B8 + ACT) * du.abs()
            val["dx"][lo:hi] = dg @ G.T.contiguous() + du @ U.T.contiguous()
            err["dx"][lo:hi] = ((edg + _gam(2 * I) * dg.abs()) @ G.T.contiguous().abs()
                                + (edu + _gam(2 * I) * du.abs()) @ U.T.contiguous().abs())
            val["dWg"][e] = X.T.contiguous() @ dg
            err["dWg"][e] = X.T.contiguous().abs() @ (edg + _gam(n) * dg.abs())
        else:
            r = u.clamp(min=0)
            h = r * r
            eh = 2 * r * eu + eu * eu + (B8 + ACT) * h
            du = dh * 2 * r
            edu = 2 * r * edh + 2 * dh.abs() * eu + (B8 + ACT) * du.abs()
            val["dx"][lo:hi] = du @ U.T.contiguous()
            err["dx"][lo:hi] = (edu + _gam(I) * du.abs()) @ U.T.contiguous().abs()
        val["y"][lo:hi] = h @ Dn
        err["y"][lo:hi] = (eh + _gam(I) * h.abs()) @ Dn.abs()
        val["dWu"][e] = X.T.contiguous() @ du
        err["dWu"][e] = X.T.contiguous().abs() @ (edu + _gam(n) * du.abs())
        val["dWd"][e] = h.T.contiguous() @ Y
        err["dWd"][e] = (eh + _gam(n) * h.abs()).T.contiguous() @ Y.abs()
    return val, {k: e + B8 * val[k].abs() + 1e-30 for k, e in err.items()}


def _check(name, got, val, err):
    d = (got.double() - val).abs()
    bad = d > 1.01 * err
    assert not bad.any(), f"{name}: {int(bad.sum())} outputs past their bound, first at {bad.nonzero()[0].tolist()}"
    norm = val.norm()
    if norm > 0 and val.numel() >= 1024:
        rel = float(d.norm() / norm)
        assert rel <= 1.1 * math.sqrt(2.0 / 3.0) * B8, f"{name}: relative error {rel:.2e}"


def _run(C, x, dy, Wg, Wu, Wd, off, act):
    y, saved = C.ffn_forward(x, Wg, Wu, Wd, offsets=off, act=act, save=True)
    y0 = C.ffn_forward(x, Wg, Wu, Wd, offsets=off, act=act)
    dx, dWg, dWu, dWd = C.ffn_backward(dy, x, Wg, Wu, Wd, saved, offsets=off, act=act)
    torch.cuda.synchronize()
    return y, y0, saved, {"y": y, "dx": dx, "dWu": dWu, "dWd": dWd, **({"dWg": dWg} if Wg is not None else {})}


# one group: lengths from one row, odd sizes around the tiles, I an odd multiple of 32
DENSE = [
    (1, 256, 128, "silu_glu"), (1, 2048, 1408, "silu_glu"), (2, 64, 32, "silu_glu"), (7, 128, 96, "relu2_up"),
    (16, 512, 384, "silu_glu"), (17, 512, 352, "silu_glu"), (33, 256, 128, "silu_glu"), (63, 320, 224, "silu_glu"),
    (64, 576, 160, "relu2_up"), (65, 1024, 512, "silu_glu"), (130, 704, 1056, "silu_glu"), (255, 256, 288, "relu2_up"),
    (257, 832, 544, "silu_glu"), (600, 2048, 768, "silu_glu"), (1000, 448, 2080, "relu2_up"), (2049, 1024, 736, "silu_glu"),
    # more tiles than fit the chip at once, and a last round that does not fill it
    (8200, 2560, 288, "silu_glu"), (8200, 2560, 224, "relu2_up"), (3000, 640, 4128, "silu_glu"),
]


@pytest.mark.parametrize("N,H,I,act", DENSE)
def test_one_group(C, N, H, I, act):
    _say(f"[ffn] N={N} H={H} I={I} {act}")
    x, dy, Wg, Wu, Wd, _ = _inputs(N, 1, H, I, act, seed=N)
    y, y0, _, got = _run(C, x, dy, Wg, Wu, Wd, None, act)
    val, err = _oracle(x, dy, Wg, Wu, Wd, [(0, N)])
    for k in got:
        _check(k, got[k], val[k], err[k])
    _check("y without kept activations", y0, val["y"], err["y"])


# row groups: (H, I, act, rows of every group, rows before the first, rows after the last)
GROUPS = [
    (256, 128, "silu_glu", [3, 0, 1, 5], 0, 0),
    (128, 32, "silu_glu", [0, 0, 0], 0, 4),
    (128, 64, "relu2_up", [1], 2, 3),
    (512, 352, "silu_glu", [0, 257, 0, 0, 63, 64, 65, 0], 0, 0),
    (320, 224, "silu_glu", [17, 300, 0, 129, 1], 5, 11),
    (448, 288, "relu2_up", [0, 255, 256, 1, 40], 3, 70),
    (2048, 768, "silu_glu", [64] * 16, 0, 0),
    (256, 96, "silu_glu", [(7 * e) % 13 for e in range(150)], 0, 1),
    (192, 64, "relu2_up", [1] * 300, 0, 0),
]


@pytest.mark.parametrize("H,I,act,counts,first,rest", GROUPS)
def test_groups(C, H, I, act, counts, first, rest):
    E, N = len(counts), first + sum(counts) + rest
    _say(f"[ffn] groups E={E} N={N} H={H} I={I} {act}")
    x, dy, Wg, Wu, Wd, off = _inputs(N, E, H, I, act, seed=E, counts=counts, first=first)
    # rows in no group hold NaN, and what is written for them stays as it was
    for t in (x, dy):
        t[:first] = float("nan")
        t[N - rest:] = float("nan")
    mark = torch.full((N, H), 7.0, dtype=torch.bfloat16, device="cuda")
    y, dx = mark.clone(), mark.clone()
    keep = (torch.full((N, I), 7.0, device="cuda") if act == "silu_glu" else None,
            torch.full((N, I), 7.0, device="cuda"), torch.full((N, I), 7.0, dtype=torch.bfloat16, device="cuda"))
    C.ffn_forward(x, Wg, Wu, Wd, offsets=off, act=act, out=y, saved=keep)
    outs = (dx, None if Wg is None else torch.empty_like(Wg), torch.empty_like(Wu), torch.empty_like(Wd))
    C.ffn_backward(dy, x, Wg, Wu, Wd, keep, offsets=off, act=act, out=outs)
    torch.cuda.synchronize()
    inside = torch.zeros(N, dtype=torch.bool, device="cuda")
    inside[first:N - rest] = True
    for t in (y, dx, *[k for k in keep if k is not None]):
        assert (t[~inside] == 7.0).all()
    rows, lo = [], first
    for c in counts:
        rows.append((lo, lo + c))
        lo += c
    val, err = _oracle(torch.where(inside[:, None], x, 0), torch.where(inside[:, None], dy, 0), Wg, Wu, Wd, rows)
    got = {"y": y, "dx": dx, "dWu": outs[2], "dWd": outs[3], **({"dWg": outs[1]} if Wg is not None else {})}
    for k, t in got.items():
        if k in ("y", "dx"):
            _check(k, t[inside], val[k][inside], err[k][inside])
        else:
            _check(k, t, val[k], err[k])
            for e, (lo, hi) in enumerate(rows):
                if lo == hi:
                    assert (t[e] == 0).all()


@pytest.mark.parametrize("N,E", [(1, 1), (40, 1), (300, 1), (300, 3)])
def test_small_whole_numbers_are_exact(C, N, E):
    """With entries in {-1, 0, 1} and few of them every intermediate is a whole
    number that bf16 holds, so the outputs are exact."""
    H, I = 192, 96
    g = torch.Generator().manual_seed(N + E)

    def few(shape, n):
        t = torch.zeros(shape)
        idx = torch.randint(0, t.shape[-1], (*t.shape[:-1], n), generator=g)
        return t.scatter_(-1, idx, torch.randint(0, 2, idx.shape, generator=g).float() * 2 - 1).bfloat16().cuda()

    x, dy = few((N, H), 3), few((N, H), 2)
    Wu, Wd = few((E, H, I), 4), few((E, I, H), 4)
    cut = [0] + [N * (e + 1) // E for e in range(E)]
    off = torch.tensor(cut, dtype=torch.int32, device="cuda")
    y, saved = C.ffn_forward(x, None, Wu, Wd, offsets=off, act="relu2_up", save=True)
    dx, _, dWu, dWd = C.ffn_backward(dy, x, None, Wu, Wd, saved, offsets=off, act="relu2_up")
    for e in range(E):
        r = slice(cut[e], cut[e + 1])
        X, U, D, Y = (t.double() for t in (x[r], Wu[e], Wd[e], dy[r]))
        u = (X @ U).clamp(min=0)
        du = (Y @ D.T.contiguous()) * 2 * u
        for name, got, want in (("up", saved[1][r], X @ U), ("hidden", saved[2][r], u * u), ("y", y[r], u * u @ D),
                                ("dx", dx[r], du @ U.T.contiguous()), ("dWu", dWu[e], X.T.contiguous() @ du),
                                ("dWd", dWd[e], (u * u).T.contiguous() @ Y)):
            assert torch.equal(got.double(), want.to(got.dtype).double()), name


def test_gradient_against_differences(C):
    """d/dt of sum(y * dy) along random directions of x and the weights, by central
    differences of the float64 formula, against the kernel's gradients."""
    N, H, I = 50, 128, 96
    x, dy, Wg, Wu, Wd, _ = _inputs(N, 1, H, I, "silu_glu", seed=5)
    _, saved = C.ffn_forward(x, Wg, Wu, Wd, save=True)
    grads = C.ffn_backward(dy, x, Wg, Wu, Wd, saved)

    def f(x, Wg, Wu, Wd):
        g, u = x @ Wg[0], x @ Wu[0]
        return float((((g * torch.sigmoid(g) * u) @ Wd[0]) * dy.double()).sum())

    at = [t.double() for t in (x, Wg, Wu, Wd)]
    gen = torch.Generator(device="cuda").manual_seed(9)
    for i, gr in enumerate(grads):
        v = torch.randn(at[i].shape, generator=gen, device="cuda", dtype=torch.float64)
        eps = 1e-5
        up, dn = list(at), list(at)
        up[i], dn[i] = at[i] + eps * v, at[i] - eps * v
        want = (f(*up) - f(*dn)) / (2 * eps)
        got = float((gr.double() * v).sum())
        # each gradient is off by two independent roundings: 2^-8 sqrt(2/3) of its
        # norm, spread over directions; five times that is past chance
        assert abs(got - want) <= 5 * math.sqrt(2 / 3) * B8 * float((gr.double() * v).norm()) + 1e-5 * abs(want)


def test_extreme_values(C):
    """Saturated gates, zero rows, and a row of infinities or NaN that stays its own."""
    H, I, N = 256, 96, 40
    x, dy, Wg, Wu, Wd, _ = _inputs(N, 1, H, I, "silu_glu", seed=3)
    x[3] *= 4096.0          # |g| in the thousands: sigmoid 0 or 1, no NaN
    x[4] = 0.0
    y, y0, _, got = _run(C, x, dy, Wg, Wu, Wd, None, "silu_glu")
    val, err = _oracle(x, dy, Wg, Wu, Wd, [(0, N)])
    for k in got:
        _check(k, got[k], val[k], err[k])
    assert (y[4] == 0).all()
    x[7, 5], x[9, 1] = float("inf"), float("nan")
    y2, _ = C.ffn_forward(x, Wg, Wu, Wd, save=True)
    clean = [i for i in range(N) if i not in (7, 9)]
    assert torch.equal(y2[clean], y[clean]) and not torch.isfinite(y2[[7, 9]]).any()


def test_offsets_outside_are_cut(C):
    """Offsets beyond the rows, or decreasing: nothing outside the tensors is
    touched, and groups whose ranges are sound are right."""
    H, I, N = 128, 64, 70
    x, dy, Wg, Wu, Wd, _ = _inputs(N, 3, H, I, "silu_glu", seed=8)
    off = torch.tensor([-5, 20, 50, 1000], dtype=torch.int32, device="cuda")
    good = torch.tensor([0, 20, 50, 70], dtype=torch.int32, device="cuda")
    for a, b in zip(_run(C, x, dy, Wg, Wu, Wd, off, "silu_glu")[3].values(),
                    _run(C, x, dy, Wg, Wu, Wd, good, "silu_glu")[3].values()):
        assert torch.equal(a, b)
    off = torch.tensor([0, 20, 10, 20], dtype=torch.int32, device="cuda")
    got = _run(C, x, dy, Wg, Wu, Wd, off, "silu_glu")[3]
    assert torch.isfinite(got["dWu"][0]).all() and (got["dWu"][1] == 0).all()


def test_repeats_and_parts(C):
    """The same bits on every call, and from calls that ask for a part."""
    x, dy, Wg, Wu, Wd, off = _inputs(500, 4, 320, 224, "silu_glu", seed=4, counts=[100, 0, 333, 67])
    _, _, saved, a = _run(C, x, dy, Wg, Wu, Wd, off, "silu_glu")
    b = _run(C, x, dy, Wg, Wu, Wd, off, "silu_glu")[3]
    assert all(torch.equal(a[k], b[k]) for k in a)
    dx, g, u, d = C.ffn_backward(dy, x, Wg, Wu, Wd, saved, offsets=off, need_dw=False)
    assert g is None and u is None and d is None and torch.equal(dx, a["dx"])
    dx, g, u, d = C.ffn_backward(dy, x, Wg, Wu, Wd, saved, offsets=off, need_dx=False)
    assert dx is None and torch.equal(g, a["dWg"]) and torch.equal(u, a["dWu"]) and torch.equal(d, a["dWd"])
    only = torch.empty_like(Wd)
    C.ffn_backward(dy, x, Wg, Wu, Wd, saved, offsets=off, out=(None, None, None, only))
    assert torch.equal(only, a["dWd"])


def test_rows_of_other_groups_stay_out(C):
    """NaN in one group's rows reaches neither another group's outputs nor its gradients."""
    H, I, counts = 192, 96, [70, 5, 130, 60]
    x, dy, Wg, Wu, Wd, off = _inputs(265, 4, H, I, "silu_glu", seed=6, counts=counts)
    want = _run(C, x, dy, Wg, Wu, Wd, off, "silu_glu")[3]
    x[70:75] = float("nan")
    dy[205:] = float("inf")
    got = _run(C, x, dy, Wg, Wu, Wd, off, "silu_glu")[3]
    for k in want:
        if k in ("y", "dx"):
            assert torch.equal(got[k][:70], want[k][:70]) and torch.equal(got[k][75:205], want[k][75:205])
        else:
            assert torch.equal(got[k][0], want[k][0]) and torch.equal(got[k][2], want[k][2])


def test_refusals(C):
    x, dy, Wg, Wu, Wd, off = _inputs(8, 2, 128, 64, "silu_glu", seed=1, counts=[3, 5])
    with pytest.raises(ValueError):
        C.ffn_forward(x, Wg, Wu, Wd)                                   # offsets missing
    with pytest.raises(ValueError):
        C.ffn_forward(x, Wg, Wu, Wd, offsets=off.long())
    with pytest.raises(ValueError):
        C.ffn_forward(x, Wg, Wu, Wd.transpose(1, 2), offsets=off)
    with pytest.raises(ValueError):
        C.ffn_forward(x[:, :64], Wg, Wu, Wd, offsets=off)
    with pytest.raises(ValueError):
        C.ffn_forward(x.float(), Wg, Wu, Wd, offsets=off)
    with pytest.raises(C.CardanError):
        C.ffn_forward(x, Wg, Wu, Wd, offsets=off, ws=torch.empty(16, dtype=torch.uint8, device="cuda"))
    _, saved = C.ffn_forward(x, Wg, Wu, Wd, offsets=off, save=True)
    with pytest.raises(ValueError):
        C.ffn_backward(dy, x, Wg, Wu, Wd, (None, *saved[1:]), offsets=off)
    with pytest.raises(C.CardanError):
        C.ffn_backward(dy, x, Wg, Wu, Wd, saved, offsets=off, need_dx=False, need_dw=False)


def test_no_rows(C):
    x, dy, Wg, Wu, Wd, _ = _inputs(0, 1, 128, 64, "silu_glu", seed=1)
    y, _, _, got = _run(C, x, dy, Wg, Wu, Wd, None, "silu_glu")
    assert y.shape == (0, 128) and all((got[k] == 0).all() for k in ("dWg", "dWu", "dWd"))


@pytest.mark.parametrize("N,E", [(3, 1), (300, 1), (300, 4)])
def test_streams_and_graphs(C, N, E):
    """A side stream and a captured graph give the eager call's bits; two graphs
    with workspaces of their own replay in any order, with eager work between."""
    H, I = 320, 224
    counts = None if E == 1 else [N // E] * E
    x, dy, Wg, Wu, Wd, off = _inputs(N, E, H, I, "silu_glu", seed=2, counts=counts)
    want = _run(C, x, dy, Wg, Wu, Wd, off, "silu_glu")[3]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _run(C, x, dy, Wg, Wu, Wd, off, "silu_glu")[3]
    side.synchronize()
    assert all(torch.equal(want[k], got[k]) for k in want)

    graphs, outs = [], []
    for _ in range(2):
        ws = torch.empty(C.ffn_workspace_bytes(C.ffn_shape(H, I, E), N), dtype=torch.uint8, device="cuda")
        y, (g, u, h) = torch.empty_like(x), (torch.empty((N, I), device="cuda"), torch.empty((N, I), device="cuda"),
                                             torch.empty((N, I), dtype=torch.bfloat16, device="cuda"))
        o = (torch.empty_like(x), torch.empty_like(Wg), torch.empty_like(Wu), torch.empty_like(Wd))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            C.ffn_forward(x, Wg, Wu, Wd, offsets=off, out=y, saved=(g, u, h), ws=ws)
            C.ffn_backward(dy, x, Wg, Wu, Wd, (g, u, h), offsets=off, ws=ws, out=o)
        graphs.append(graph)
        outs.append(dict(y=y, dx=o[0], dWg=o[1], dWu=o[2], dWd=o[3]))
    for step in range(3):
        for graph, o in zip(graphs, outs):
            for t in o.values():
                t.fill_(3.0)
            graph.replay()
        C.ffn_forward(x, Wg, Wu, Wd, offsets=off)
        torch.cuda.synchronize()
        for o in outs:
            assert all(torch.equal(want[k], o[k]) for k in want), step
