"""Where the arrays of the distillation loss may start (CPU only: every call
fails validation, or has no rows; the fake pointers are never dereferenced)."""

import pytest

FAKE = 0x10000
ANY = 16


@pytest.fixture(scope="module")
def C():
    import os

    from paper_2609_21137_amd import build
    if not os.path.exists(build.LIB):
        build.build()
    from paper_2609_21137_amd import cardan
    return cardan


def _call(C, typ, N=2, K=4, logits=FAKE, teacher=FAKE, ids=FAKE, loss=FAKE, d=FAKE + 4096, T=1.0, dld=100):
    rc = C.lib().cardan_distill_loss(N, 100, K, typ, logits, 100, teacher, ids, None, T, 0.0, None, loss, d, dld, None)
    return rc, C.lib().cardan_last_error().decode()


def test_any_element(C):
    # (the last array fails, so that no call is launched)
    for typ, size in ((ANY, 2), (ANY + 1, 4)):
        for at in range(size, 16, size):
            rc, msg = _call(C, typ, logits=FAKE + at, loss=FAKE + 4, teacher=FAKE + 4, ids=FAKE + 12, d=FAKE + 4097)
            assert rc == -6 and msg.startswith("dlogits"), msg


@pytest.mark.parametrize("name,off", [("logits", 1), ("teacher", 2), ("ids", 1), ("loss", 2), ("d", 1)])
def test_refusals(C, name, off):
    assert _call(C, ANY, **{name: FAKE + off})[0] == -6
    assert _call(C, 0, **{name: FAKE + 8 + (off & 1)})[0] == -6      # without the flag: 16 bytes
    if name != "d":
        assert _call(C, ANY, **{name: None})[0] == -1
    if name == "logits":
        assert _call(C, ANY + 1, logits=FAKE + 2)[0] == -6


def test_types(C):
    for typ in (2, ANY + 2, 2 * ANY, -1, -ANY):
        assert _call(C, typ)[0] == -3
    assert _call(C, ANY, T=0.0)[0] == -2
    assert _call(C, ANY, N=0, logits=None, teacher=None, ids=None, loss=None, d=None)[0] == 0
