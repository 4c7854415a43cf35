"""A NaN stays one through the feed-forward block, with either activation.

The comparisons are exact: a row with NaN in x or dy has NaN in every output of
its own that its formulas reach, rows beside it keep their bits. Weights have no
zeros, so each element of a row's projections is NaN.
"""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def C():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_21137_amd import cardan
    return cardan


def _inputs(N, E, H, I, act, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def n(*shape, std=1.0):
        t = (torch.randn(shape, generator=g, device="cuda") * std).to(torch.bfloat16)
        return torch.where(t == 0, std, t)

    return (n(N, H), n(N, H, std=0.1), n(E, H, I, std=H ** -0.5) if act == "silu_glu" else None,
            n(E, H, I, std=H ** -0.5), n(E, I, H, std=I ** -0.5))


# few rows without and with parts of the sum, few rows in several blocks, tiles, tiles of row groups
@pytest.mark.parametrize("N,H,I,groups", [(3, 256, 128, 0), (9, 2048, 1408, 0), (40, 256, 96, 0), (300, 320, 224, 0),
                                          (300, 320, 224, 3)])
@pytest.mark.parametrize("act", ["silu_glu", "relu2_up"])
def test_a_row_of_nan_is_seen(C, act, N, H, I, groups):
    print(f"[ffn nan] {act} N={N} H={H} I={I} groups={groups}", flush=True)
    E = max(1, groups)
    x, dy, Wg, Wu, Wd = _inputs(N, E, H, I, act, N)
    off = torch.arange(E + 1, device="cuda", dtype=torch.int32) * (N // E) if groups else None
    bad = N - 2                                           # (in the last group)
    rest = [n for n in range(N) if n != bad]

    def run():
        y, saved = C.ffn_forward(x, Wg, Wu, Wd, offsets=off, act=act, save=True)
        alone = C.ffn_forward(x, Wg, Wu, Wd, offsets=off, act=act)
        return (y, alone, saved, *C.ffn_backward(dy, x, Wg, Wu, Wd, saved, offsets=off, act=act))

    y0, alone0, _, dx0, *dW0 = run()
    x[bad, 5] = float("nan")
    y, alone, (_, u, h), dx, *dW = run()
    torch.cuda.synchronize()
    for t in (u, h, y, alone, dx):
        assert torch.isnan(t[bad]).all()
    for t, t0 in ((y, y0), (alone, alone0), (dx, dx0)):
        assert torch.equal(t[rest], t0[rest])
    for t, t0 in zip(dW, dW0):
        if t is None:
            continue
        assert torch.equal(t[:E - 1], t0[:E - 1]) and torch.isnan(t[E - 1]).any()
    assert torch.isnan(dW[2][E - 1]).all()                # h^T dy: each of its sums has the row


@pytest.mark.parametrize("N", [33, 300])
@pytest.mark.parametrize("act", ["silu_glu", "relu2_up"])
def test_a_gradient_of_nan_is_seen(C, act, N):
    x, dy, Wg, Wu, Wd = _inputs(N, 1, 256, 128, act, 5)
    _, saved = C.ffn_forward(x, Wg, Wu, Wd, act=act, save=True)
    dy[2, 7] = float("nan")
    dx, _, dWu, dWd = C.ffn_backward(dy, x, Wg, Wu, Wd, saved, act=act)
    torch.cuda.synchronize()
    rest = [n for n in range(N) if n != 2]
    assert torch.isnan(dx[2]).all() and torch.isfinite(dx[rest]).all()
    assert torch.isnan(dWu).all() and torch.isnan(dWd[..., 7]).all()
