"""Sizes past 32 bits are refused, not cut to their low bits (CPU only)."""

import os

import pytest
import torch

PAST = 1 << 32


@pytest.fixture(scope="module")
def C():
    from paper_2609_21137_amd import build
    if not os.path.exists(build.LIB):
        build.build()
    from paper_2609_21137_amd import cardan
    return cardan


def test_workspaces(C):
    for N in (PAST, PAST + 1, PAST + 65, 1 << 31, 1 << 40):
        with pytest.raises(ValueError, match="32 bits"):
            C.route_rows_workspace_bytes(N, 64, 4)
        with pytest.raises(ValueError, match="32 bits"):
            C.ffn_workspace_bytes(C.ffn_shape(64, 64), N)
    with pytest.raises(C.CardanError):
        C.route_rows_workspace_bytes(-1, 64, 4)
    with pytest.raises(C.CardanError):
        C.route_rows_workspace_bytes((1 << 30) + 1, 64, 4)


@pytest.mark.parametrize("name", ["E", "top_k", "groups", "top_groups", "group_best"])
def test_routings(C, name):
    kw = dict(E=64, top_k=4, score="softmax", renorm=True, scale=1.0, groups=1, top_groups=1, group_best=1)
    kw[name] += PAST
    with pytest.raises(ValueError, match="32 bits"):
        C.route_rows_workspace_bytes(8, **kw)


def _rows(n, w, dtype):
    """A tensor of n rows whose memory is never touched."""
    return torch.empty((n, w), dtype=dtype, device="meta")


def test_rows(C):
    """The sizes are looked at before the tensors, which live on no GPU here."""
    bf, i32, f32, N = torch.bfloat16, torch.int32, torch.float32, PAST + 3
    small, place = torch.zeros((2, 8), dtype=bf), torch.zeros((2, 2), dtype=i32)
    for call in (lambda: C.dispatch_rows(_rows(N, 1, bf), _rows(N, 1, i32)),
                 lambda: C.dispatch_rows(small, place, rows=N),
                 lambda: C.dispatch_rows(small, place, out=_rows(N, 8, bf)),
                 lambda: C.combine_rows(_rows(N, 8, bf), place),
                 lambda: C.combine_rows(small, _rows(N, 2, i32)),
                 lambda: C.combine_rows_backward(small, _rows(N, 8, bf), place),
                 lambda: C.combine_rows_backward(_rows(N, 8, bf), small, _rows(N, 2, i32))):
        with pytest.raises(ValueError, match="32 bits"):
            call()


def test_steps(C):
    p = torch.zeros(8)
    for step in (PAST + 1, 1 << 31, -PAST + 1):
        with pytest.raises(ValueError, match="32 bits"):
            C.adamw_step([p], [p], [C.adamw_state(p)], step, 1e-3)
