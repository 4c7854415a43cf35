"""Refusals of the routing of many rows, of rows to their experts and back and of
the AdamW step, on the CPU.

Every call here fails validation, or has nothing to launch, before a device call
is reached; the fake pointers are never dereferenced.
"""

import ctypes
import math
import os

import pytest
import torch

FAKE, ODD = 0x10000, 0x10001


@pytest.fixture(scope="module")
def C():
    from paper_2609_21137_amd import build
    if not os.path.exists(build.LIB):
        build.build()
    from paper_2609_21137_amd import cardan
    return cardan


def _routing(C, **kw):
    d = dict(E=64, top_k=4, score=0, renorm=1, groups=1, top_groups=1, group_best=1, scale=1.0)
    d.update(kw)
    return C.Routing(*(d[n] for n, _ in C.Routing._fields_))


BAD = [
    (dict(E=0), -3), (dict(E=1025), -3), (dict(E=-1), -3), (dict(top_k=0), -2), (dict(top_k=65), -2),
    (dict(top_k=33), -3), (dict(score=2), -3), (dict(score=-1), -3), (dict(renorm=2), -2), (dict(groups=0), -3),
    (dict(groups=65, E=130), -3), (dict(groups=3), -2), (dict(groups=4, top_groups=0), -2), (dict(groups=4, top_groups=5), -2),
    (dict(groups=32, top_groups=1), -2), (dict(groups=4, top_groups=1, group_best=0), -3),
    (dict(groups=4, top_groups=1, group_best=3), -3), (dict(groups=64, top_groups=4, group_best=2), -2),
    (dict(scale=math.inf), -2), (dict(scale=math.nan), -2),
]


@pytest.mark.parametrize("kw,code", BAD)
def test_bad_routings(C, kw, code):
    r, n = _routing(C, **kw), ctypes.c_size_t(0)
    lib = C.lib()
    assert lib.cardan_route_rows_workspace_bytes(ctypes.byref(r), 8, ctypes.byref(n)) == code and lib.cardan_last_error()
    assert lib.cardan_route_rows(ctypes.byref(r), 8, 1, FAKE, 4096, None, FAKE, FAKE, None, None, None, 0, None) == code
    assert lib.cardan_route_rows_backward(ctypes.byref(r), 8, 1, FAKE, 4096, FAKE, FAKE, FAKE, 4096, None) == code


def test_route_workspace(C):
    lib, n = C.lib(), ctypes.c_size_t(0)
    assert lib.cardan_route_rows_workspace_bytes(None, 1, ctypes.byref(n)) == -1
    r = _routing(C)
    assert lib.cardan_route_rows_workspace_bytes(ctypes.byref(r), 1, None) == -1
    for N, code in ((-1, -2), ((1 << 30) + 1, -2), (1 << 29, -3)):
        assert lib.cardan_route_rows_workspace_bytes(ctypes.byref(r), N, ctypes.byref(n)) == code
    sizes = [C.route_rows_workspace_bytes(N, 64, 4) for N in (0, 1, 64, 65, 1000, 4096, 100000, (1 << 29) - 1)]
    assert sizes == sorted(sizes) and sizes[0] == 0
    # counts of 16 bits for blocks of 32 rows (16 above 128 experts, 4 above 256), of at most 256
    # blocks, or more where a block would have more than 2^15 rows
    for E, rows in ((64, 32), (200, 16), (301, 4)):
        for N in (65, 66, 1000, 5000, 1 << 20, 1 << 24, (1 << 29) - 1):
            blocks = max(min(256, -(-N // rows)), -(-N >> 15))
            assert C.route_rows_workspace_bytes(N, E, 4) >= blocks * E * 2


def _route(C, N=100, kind=1, logits=FAKE, ld=64, bias=None, idx=FAKE, w=FAKE, place=FAKE, off=FAKE, ws=FAKE, nbytes=None, **kw):
    r, n = _routing(C, **kw), ctypes.c_size_t(0)
    C.lib().cardan_route_rows_workspace_bytes(ctypes.byref(r), max(N, 0), ctypes.byref(n))
    return C.lib().cardan_route_rows(ctypes.byref(r), N, kind, logits, ld, bias, idx, w, place, off, ws,
                                     n.value if nbytes is None else nbytes, None)


def test_route_refusals(C):
    assert C.lib().cardan_route_rows(None, 1, 1, FAKE, 64, None, FAKE, FAKE, None, None, None, 0, None) == -1
    assert _route(C, N=-1) == -2 and _route(C, kind=3) == -3 and _route(C, kind=-1) == -3 and _route(C, kind=17) == -3
    assert _route(C, ld=63) == -2 and _route(C, ld=(1 << 40) + 1) == -2
    for name in ("logits", "idx", "w", "place", "off", "ws"):
        assert _route(C, **{name: None}) == -1, name
    for name in ("logits", "bias", "idx", "w", "place", "off", "ws"):
        assert _route(C, **{name: ODD}) == -6, name
    assert _route(C, kind=0, logits=FAKE + 2, ws=None) == -1       # (bf16 rows may start on 2 bytes)
    assert _route(C, kind=2, logits=FAKE + 4) == -6
    assert _route(C, nbytes=C.route_rows_workspace_bytes(100, 64, 4) - 1) == -4
    assert _route(C, nbytes=0) == -4


def _back(C, N=100, kind=1, logits=FAKE, ld=64, idx=FAKE, d=FAKE, out=FAKE * 2, dld=64, **kw):
    r = _routing(C, **kw)
    return C.lib().cardan_route_rows_backward(ctypes.byref(r), N, kind, logits, ld, idx, d, out, dld, None)


def test_route_backward_refusals(C):
    assert _back(C, N=-1) == -2 and _back(C, kind=3) == -3 and _back(C, ld=63) == -2 and _back(C, dld=63) == -2
    assert _back(C, dld=(1 << 40) + 1) == -2 and _back(C, out=FAKE, dld=65) == -2
    for name in ("logits", "idx", "d", "out"):
        assert _back(C, **{name: None}) == -1, name
        assert _back(C, **{name: ODD}) == -6, name
    assert _back(C, N=0, logits=None, idx=None, d=None, out=None) == 0


def test_rows_refusals(C):
    lib = C.lib()

    def dispatch(N=4, k=2, H=64, M=8, x=FAKE, place=FAKE, xe=FAKE):
        return lib.cardan_dispatch_rows(N, k, H, M, x, place, xe, None)

    def combine(N=4, k=2, H=64, M=8, ye=FAKE, place=FAKE, w=None, kind=0, y=FAKE):
        return lib.cardan_combine_rows(N, k, H, M, ye, place, w, kind, y, None)

    def back(N=4, k=2, H=64, M=8, kind=0, dy=FAKE, ye=FAKE, place=FAKE, w=None, dye=FAKE, dw=FAKE):
        return lib.cardan_combine_rows_backward(N, k, H, M, kind, dy, ye, place, w, dye, dw, None)

    for f in (dispatch, combine, back):
        for kw, code in ((dict(N=-1), -2), (dict(N=(1 << 30) + 1), -2), (dict(M=-1), -2), (dict(k=0), -3), (dict(k=33), -3),
                         (dict(H=0), -3), (dict(H=(1 << 20) + 1), -3), (dict(place=None), -1), (dict(place=ODD + 1), -6)):
            assert f(**kw) == code, (f, kw)
        assert f(N=0, place=None) == 0
    assert dispatch(x=None) == -1 and dispatch(xe=None) == -1 and dispatch(x=ODD) == -6 and dispatch(xe=ODD) == -6
    assert dispatch(M=0, xe=None) == 0
    assert combine(ye=None) == -1 and combine(y=None) == -1 and combine(kind=2) == -3 and combine(w=ODD + 1) == -6
    assert combine(kind=1, y=FAKE + 2) == -6 and combine(ye=ODD) == -6
    assert back(dy=None) == -1 and back(ye=None) == -1 and back(dye=None, dw=None) == -1 and back(kind=2) == -3
    assert back(kind=1, dy=FAKE + 2) == -6 and back(dw=FAKE + 2) == -6 and back(dye=ODD) == -6 and back(w=FAKE + 2) == -6
    assert back(M=0, dye=None, dw=None) == 0


def _adamw(C, tensors=1, conf=None, **kw):
    base = dict(param=FAKE, grad=FAKE, m=FAKE, v=FAKE, m_scale=None, v_scale=None, copy=None, n=100)
    base.update(kw)
    t = (C.AdamwTensor * max(1, tensors))(*(C.AdamwTensor(**base) for _ in range(max(1, tensors))))
    c = dict(param_type=1, grad_type=1, state_bits=32, step=1, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0,
             step_device=None, lr_device=None, grad_scale=None)
    c.update(conf or {})
    return C.lib().cardan_adamw_step(ctypes.byref(C.Adamw(**c)), tensors, t, None)


@pytest.mark.parametrize("conf,code", [
    (dict(param_type=2), -3), (dict(grad_type=-1), -3), (dict(state_bits=16), -3), (dict(step=0), -2), (dict(step=-5), -2),
    (dict(beta1=1.0), -2), (dict(beta1=-0.1), -2), (dict(beta2=1.0), -2), (dict(beta2=math.nan), -2), (dict(eps=-1e-8), -2),
    (dict(eps=math.inf), -2), (dict(eps=math.nan), -2), (dict(lr=math.inf), -2), (dict(weight_decay=math.nan), -2),
    (dict(step_device=FAKE + 2), -6), (dict(lr_device=FAKE + 1), -6), (dict(grad_scale=FAKE + 3), -6),
])
def test_adamw_bad_settings(C, conf, code):
    assert _adamw(C, conf=conf) == code and C.lib().cardan_last_error()


def test_adamw_refusals(C):
    lib = C.lib()
    assert lib.cardan_adamw_step(None, 0, None, None) == -1
    assert _adamw(C, tensors=-1) == -2
    c = C.Adamw(1, 1, 32, 1, 1e-3, 0.9, 0.999, 1e-8, 0.0)
    assert lib.cardan_adamw_step(ctypes.byref(c), 1, None, None) == -1
    assert lib.cardan_adamw_step(ctypes.byref(c), 0, None, None) == 0
    assert _adamw(C, n=-1) == -2 and _adamw(C, n=(1 << 34) + 1) == -2
    assert _adamw(C, n=0, param=None, grad=None, m=None, v=None) == 0
    for name in ("param", "grad", "m", "v"):
        assert _adamw(C, **{name: None}) == -1, name
        assert _adamw(C, **{name: ODD}) == -6, name
    assert _adamw(C, copy=ODD) == -6
    eight = dict(state_bits=8)
    assert _adamw(C, conf=eight) == -1
    assert _adamw(C, conf=eight, m_scale=FAKE, v_scale=FAKE + 2) == -6
    assert _adamw(C, conf=eight, m=ODD, v=ODD, m_scale=FAKE, v_scale=None) == -1
    assert _adamw(C, conf=dict(param_type=0), copy=FAKE) == -3
    # every tensor of a call is looked at before any is launched
    t = (C.AdamwTensor * 50)(*(C.AdamwTensor(FAKE, FAKE, FAKE, FAKE, None, None, None, 10) for _ in range(50)))
    t[49].grad = None
    assert lib.cardan_adamw_step(ctypes.byref(c), 50, t, None) == -1


def test_binding_refuses(C):
    """Host tensors, other types and shapes raise before the library is called."""
    z = torch.zeros(4, 8)
    i2 = torch.zeros(4, 2, dtype=torch.int32)
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        C.route_rows(z, 2)
    with pytest.raises(ValueError):
        C.route_rows(z.to(torch.float16), 2)
    with pytest.raises(ValueError):
        C.route_rows(z[0], 2)
    with pytest.raises(ValueError):
        C.route_rows_backward(z, i2, torch.zeros(4, 2))
    with pytest.raises(ValueError):
        C.route_rows_backward(z, i2, torch.zeros(4, 2), top_k=3)
    with pytest.raises(ValueError):
        C._routing(8, 2, "tanh", True, 1.0, 1, 1, 1)
    with pytest.raises(ValueError):
        C.dispatch_rows(x, i2)
    with pytest.raises(ValueError):
        C.combine_rows(x, i2)
    with pytest.raises(ValueError):
        C.combine_rows_backward(x, x, i2)
    p = torch.zeros(8)
    with pytest.raises(ValueError):
        C.adamw_step([p], [p], [C.adamw_state(p)], 1, 1e-3)
    with pytest.raises(ValueError):
        C.adamw_step([p], [], [], 1, 1e-3)
    with pytest.raises(ValueError):
        C.adamw_step([p.double()], [p], [C.adamw_state(p)], 1, 1e-3)
    with pytest.raises(ValueError):
        C.adamw_step([p], [p], [(p,)], 1, 1e-3)
    with pytest.raises(ValueError):
        C.adamw_state(p, 16)
    C.adamw_step([], [], [], 1, 1e-3)


def test_states(C):
    p = torch.zeros(3, 100)
    m, v = C.adamw_state(p)
    assert m.shape == v.shape == (3, 100) and m.dtype == v.dtype == torch.float32
    m, v, ms, vs = C.adamw_state(p, 8)
    assert m.dtype is torch.float8_e4m3fn and v.dtype is torch.float8_e5m2 and ms.shape == vs.shape == (2,)
