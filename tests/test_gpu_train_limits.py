"""Calls of the feed-forward block and the distillation loss at the ends of what
they take: offsets out of order, rows past one launch, arrays past 2^31 elements.

Bounds: those of tests/test_gpu_ffn.py and tests/test_gpu_distill.py.
"""

import pytest
import torch
from test_gpu_distill import _check as _check_loss
from test_gpu_distill import _oracle as _loss_oracle
from test_gpu_ffn import _check, _inputs, _oracle, _run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def C():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_21137_amd import cardan
    return cardan


@pytest.fixture(autouse=True)
def _free():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("act", ["silu_glu", "relu2_up"])
def test_decreasing_offsets_leave_sound_groups_right(C, act):
    """Group 0 of [0, 20, 10, 20] is sound: its outputs and gradients are those of [0, 20, 20, 20]."""
    H, I, N = 128, 64, 70
    x, dy, Wg, Wu, Wd, _ = _inputs(N, 3, H, I, act, seed=8)
    off = torch.tensor([0, 20, 10, 20], dtype=torch.int32, device="cuda")
    good = torch.tensor([0, 20, 20, 20], dtype=torch.int32, device="cuda")
    got, want = (_run(C, x, dy, Wg, Wu, Wd, o, act)[3] for o in (off, good))
    val, err = _oracle(x, dy, Wg, Wu, Wd, [(0, 20), (20, 20), (20, 20)])
    for k in got:
        part = (slice(0, 20),) if k in ("y", "dx") else (0,)
        assert torch.equal(got[k][part], want[k][part])
        _check(k, got[k][part], val[k][part], err[k][part])
        if k not in ("y", "dx"):
            assert (got[k][1] == 0).all()


def _rows(N, V, K, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    logits = torch.empty((N, V), dtype=dtype, device="cuda").normal_(0.0, 2.0, generator=g)
    first = torch.randint(0, V, (N, 1), generator=g, device="cuda")
    ids = ((first + torch.arange(K, device="cuda")) % V).int()
    teacher = torch.randn((N, K), generator=g, device="cuda") * 3
    labels = torch.randint(0, V, (N,), generator=g, device="cuda").int()
    return logits, teacher, ids, labels, torch.randn((N,), generator=g, device="cuda")


@pytest.mark.parametrize("dtype,T", [(torch.bfloat16, 2.0), (torch.float32, 3.0)])
def test_rows_of_several_launches(C, dtype, T):
    """2^21 rows go through one launch; those behind them have their own entries."""
    N, V, K = (1 << 21) + 3, 9, 2
    print(f"[distill] N={N} V={V} {dtype}", flush=True)
    logits, teacher, ids, labels, w = _rows(N, V, K, dtype, 1)
    loss, d = C.distill_loss(logits, teacher, ids, labels=labels, temperature=T, ce_weight=0.5, row_weight=w)
    _check_loss(loss, d, _loss_oracle(logits, teacher, ids, labels, T, 0.5, w), dtype)


def test_logits_past_32_bits(C):
    """2^31 logits and more: rows on both sides of 2^31 and 2^32 bytes and of 2^31 elements."""
    N, V, K = 32800, 65541, 40
    print(f"[distill] N={N} V={V}", flush=True)
    logits, teacher, ids, labels, w = _rows(N, V, K, torch.bfloat16, 2)
    assert logits.numel() > 1 << 31
    args = dict(temperature=2.0, ce_weight=0.5)
    loss, d = C.distill_loss(logits, teacher, ids, labels=labels, row_weight=w, **args)
    for bytes_at in (0, 1 << 31, 1 << 32, (1 << 32) + 2 * V, 2 * N * V - 1):
        n = max(0, min(N - 3, bytes_at // (2 * V) - 1))
        p = slice(n, n + 3)
        want = _loss_oracle(logits[p], teacher[p], ids[p], labels[p], 2.0, 0.5, w[p])
        _check_loss(loss[p], d[p], want, torch.bfloat16)


@pytest.mark.parametrize("H,I,act", [(4096, 32, "silu_glu"), (64, 4096, "relu2_up")])
def test_rows_past_32_bits(C, H, I, act):
    """x and y, or the hidden activations, of more than 2^31 elements."""
    N, E = 530000, 2
    print(f"[ffn] N={N} H={H} I={I} {act}", flush=True)
    assert N * max(H, I) > 1 << 31
    g = torch.Generator(device="cuda").manual_seed(3)

    def n(*shape, std=1.0):
        return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, std, generator=g)

    cut = 200001
    x, dy = n(N, H), n(N, H, std=0.1)
    Wg = n(E, H, I, std=H ** -0.5) if act == "silu_glu" else None
    Wu, Wd = n(E, H, I, std=H ** -0.5), n(E, I, H, std=I ** -0.5)
    off = torch.tensor([0, cut, N], dtype=torch.int32, device="cuda")
    y, saved = C.ffn_forward(x, Wg, Wu, Wd, offsets=off, act=act, save=True)
    dx, dWg, dWu, dWd = C.ffn_backward(dy, x, Wg, Wu, Wd, saved, offsets=off, act=act)
    torch.cuda.synchronize()
    # rows: single ones of both groups, by the oracle of 64 rows
    for lo in (0, cut - 32, (1 << 31) // (2 * max(H, I)) - 32, (1 << 31) // max(H, I) - 32, N - 64):
        p = slice(lo, lo + 64)
        a = max(0, min(64, cut - lo))
        val, err = _oracle(x[p], dy[p], Wg, Wu, Wd, [(0, a), (a, 64)])
        _check("y", y[p], val["y"], err["y"])
        _check("dx", dx[p], val["dx"], err["dx"])
    # the weights' gradients add up over calls that each take a part of the rows (float64
    # sums of their bf16 values: each part, and the whole, is off by half a step and by its terms)
    parts = [torch.zeros(t.shape, dtype=torch.float64, device="cuda") for t in (dWu, dWd)]
    step = 1 << 16
    for e, (lo, hi) in enumerate(((0, cut), (cut, N))):
        for r in range(lo, hi, step):
            p = slice(r, min(r + step, hi))
            w = [None if t is None else t[e] for t in (Wg, Wu, Wd)]
            _, kept = C.ffn_forward(x[p], *w, act=act, save=True)
            got = C.ffn_backward(dy[p], x[p], *w, kept, act=act, need_dx=False)
            parts[0][e] += got[2].double()
            parts[1][e] += got[3].double()
    for t, want in zip((dWu, dWd), parts):
        # roundings of nine values at most, of comparable size and independent: 2^-8 / sqrt(3)
        # of each, and the parts' norms add as a root of squares
        assert float((t.double() - want).norm() / want.norm()) <= 1.1 * 2.0 ** -8 * (2.0 / 3.0) ** 0.5


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [1.0, 2.0, 3.0])
def test_a_row_masked_out_whole(C, dtype, T):
    """A student's row of -inf has no softmax: NaN there, the other rows as they were."""
    logits, teacher, ids, labels, w = _rows(6, 777, 12, dtype, 4)
    args = dict(labels=labels, temperature=T, ce_weight=0.5, row_weight=w)
    loss0, d0 = C.distill_loss(logits, teacher, ids, **args)
    logits[2] = float("-inf")
    loss, d = C.distill_loss(logits, teacher, ids, **args)
    assert torch.isnan(loss[2]).all() and torch.isnan(d[2]).all()
    rest = [0, 1, 3, 4, 5]
    assert torch.equal(loss[rest], loss0[rest]) and torch.equal(d[rest], d0[rest])
