"""Refusals of the feed-forward block and the distillation loss on the CPU.

Every call here fails validation before a device call is reached; the fake
pointers are never dereferenced.
"""

import ctypes
import os
import re
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

FAKE, ODD = 0x10000, 0x10004


@pytest.fixture(scope="module")
def C():
    from paper_2609_21137_amd import build
    if not os.path.exists(build.LIB):
        build.build()
    from paper_2609_21137_amd import cardan
    return cardan


def _ffn_bytes(C, shape, N):
    n = ctypes.c_size_t(0)
    return C.lib().cardan_ffn_workspace_bytes(None if shape is None else ctypes.byref(shape), N, ctypes.byref(n)), n.value


@pytest.mark.parametrize("dims,N,code", [
    ((2048, 768, 1, 0), -1, -2), ((2048, 768, 1, 0), (1 << 30) + 1, -2), ((0, 768, 1, 0), 1, -2), ((2048, -32, 1, 0), 1, -2), ((2048, 768, 0, 0), 1, -2),
    ((2048, 768, 1, 2), 1, -3), ((2048, 768, 1, -1), 1, -3), ((2080, 768, 1, 0), 1, -3), ((2048, 784, 1, 0), 1, -3),
    ((2048, 768, 1025, 0), 1, -3), ((32768, 32768, 1, 0), 1, -3), ((1 << 21, 32, 1, 0), 1, -3), ((64, 1 << 21, 1, 0), 1, -3),
])
def test_ffn_bad_shapes(C, dims, N, code):
    rc, _ = _ffn_bytes(C, C.FfnShape(*dims), N)
    assert rc == code and C.lib().cardan_last_error()


def test_ffn_workspace(C):
    assert _ffn_bytes(C, None, 1)[0] == -1
    assert C.lib().cardan_ffn_workspace_bytes(ctypes.byref(C.ffn_shape(64, 32)), 1, None) == -1
    for dims in ((2048, 768, 1, 0), (2048, 768, 128, 0), (4096, 14336, 1, 1)):
        sizes = [C.ffn_workspace_bytes(C.FfnShape(*dims), N) for N in (0, 1, 16, 64, 65, 1000, 8192, 1 << 20)]
        assert all(s >= 2 * 2 * N * dims[1] for s, N in zip(sizes, (0, 1, 16, 64, 65, 1000, 8192, 1 << 20)))


def _forward(C, shape=None, N=4, x=FAKE, off=None, w=(FAKE, FAKE, FAKE), y=FAKE, keep=(None, None, None), ws=FAKE,
             nbytes=None, weights=True):
    shape = shape or C.ffn_shape(256, 128)
    st = C.FfnWeightsStruct(*w)
    need = _ffn_bytes(C, shape, max(N, 0))[1]
    return C.lib().cardan_ffn_forward(ctypes.byref(shape), N, x, off, ctypes.byref(st) if weights else None, y, *keep,
                                      ws, need if nbytes is None else nbytes, None)


def test_ffn_forward_refusals(C):
    relu2 = C.ffn_shape(256, 128, act="relu2_up")
    many = C.ffn_shape(256, 128, 4)
    assert _forward(C, N=-1) == -2
    assert _forward(C, weights=False) == -1
    assert _forward(C, w=(None, FAKE, FAKE)) == -1
    assert _forward(C, w=(FAKE, None, FAKE)) == -1
    assert _forward(C, w=(FAKE, FAKE, ODD)) == -6
    assert _forward(C, x=None) == -1
    assert _forward(C, x=ODD) == -6
    assert _forward(C, y=None) == -1
    assert _forward(C, shape=many) == -1                       # offsets missing
    assert _forward(C, shape=many, off=FAKE + 2) == -6
    assert _forward(C, keep=(None, FAKE, FAKE)) == -1
    assert _forward(C, keep=(FAKE, FAKE, None)) == -1
    assert _forward(C, keep=(FAKE, ODD, FAKE)) == -6
    assert _forward(C, shape=relu2, keep=(FAKE, FAKE, FAKE)) == -2
    assert _forward(C, ws=None) == -1
    assert _forward(C, ws=ODD) == -6
    assert _forward(C, nbytes=16) == -4
    assert _forward(C, N=0, x=None, y=None) == 0               # nothing to do


def _backward(C, shape=None, N=4, dy=FAKE, x=FAKE, off=None, w=(FAKE, FAKE, FAKE), keep=(FAKE, FAKE, FAKE),
              outs=(FAKE, FAKE, FAKE, FAKE), ws=FAKE, nbytes=None):
    shape = shape or C.ffn_shape(256, 128)
    st = C.FfnWeightsStruct(*w)
    need = _ffn_bytes(C, shape, N)[1]
    return C.lib().cardan_ffn_backward(ctypes.byref(shape), N, dy, x, off, ctypes.byref(st), *keep, *outs, ws,
                                       need if nbytes is None else nbytes, None)


def test_ffn_backward_refusals(C):
    relu2 = C.ffn_shape(256, 128, act="relu2_up")
    assert _backward(C, dy=None) == -1
    assert _backward(C, x=ODD) == -6
    assert _backward(C, keep=(None, FAKE, FAKE)) == -1
    assert _backward(C, keep=(FAKE, None, FAKE)) == -1
    assert _backward(C, keep=(FAKE, FAKE, None)) == -1
    assert _backward(C, outs=(None, None, None, None)) == -1
    assert _backward(C, outs=(FAKE, FAKE, None, FAKE)) == -1   # one of dW_gate, dW_up
    assert _backward(C, outs=(ODD, FAKE, FAKE, FAKE)) == -6
    assert _backward(C, outs=(FAKE, FAKE, FAKE, ODD)) == -6
    assert _backward(C, shape=relu2) == -2                     # gate of up-only experts
    assert _backward(C, shape=relu2, keep=(None, FAKE, FAKE)) == -2
    assert _backward(C, shape=C.ffn_shape(256, 128, 2)) == -1
    assert _backward(C, nbytes=16) == -4


def _distill(C, N=2, V=100, K=4, typ=0, logits=FAKE, ld=100, teacher=FAKE, ids=FAKE, labels=None, T=1.0, c=0.0, w=None,
             loss=FAKE, d=None, dld=0):
    return C.lib().cardan_distill_loss(N, V, K, typ, logits, ld, teacher, ids, labels, T, c, w, loss, d, dld, None)


def test_distill_refusals(C):
    inf, nan = float("inf"), float("nan")
    assert _distill(C, N=-1) == -2
    assert _distill(C, V=0) == -2
    assert _distill(C, V=(1 << 30) + 1, ld=1 << 31) == -2
    assert _distill(C, K=-1) == -3 and _distill(C, K=1025) == -3
    assert _distill(C, typ=2) == -3
    assert _distill(C, ld=99) == -2
    assert _distill(C, d=FAKE + 4096, dld=99) == -2
    assert _distill(C, d=FAKE, dld=101) == -2                  # in place with other rows
    for T in (0.0, -1.0, inf, nan, 1e-45, 2.0 ** -17, 2.0 ** 17):
        assert _distill(C, T=T) == -2
    assert _distill(C, N=(1 << 30) + 1) == -2
    assert _distill(C, c=inf) == -2 and _distill(C, c=nan) == -2
    assert _distill(C, logits=None) == -1 and _distill(C, logits=ODD) == -6
    assert _distill(C, teacher=None) == -1 and _distill(C, ids=None) == -1
    assert _distill(C, loss=None) == -1 and _distill(C, loss=ODD) == -6
    assert _distill(C, d=ODD, dld=100) == -6
    assert _distill(C, labels=FAKE + 2) == -6 and _distill(C, w=FAKE + 1) == -6
    assert _distill(C, N=0, logits=None, loss=None) == 0


def test_binding_refuses(C):
    x = torch.zeros((4, 256), dtype=torch.bfloat16)
    wu, wd = torch.zeros((256, 128), dtype=torch.bfloat16), torch.zeros((128, 256), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        C.ffn_forward(x, wu, wu, wd)                           # host tensors
    with pytest.raises(ValueError):
        C.ffn_forward(x[0], wu, wu, wd)
    with pytest.raises(ValueError):
        C.ffn_forward(x, wu, wu, wd, act="gelu")
    with pytest.raises(ValueError):
        C.ffn_forward(x, wu, wu, wd, act="relu2_up")           # W_gate of up-only experts
    z, t, i = torch.zeros((2, 10)), torch.zeros((2, 3)), torch.zeros((2, 3), dtype=torch.int32)
    with pytest.raises(ValueError):
        C.distill_loss(z, t, i)
    with pytest.raises(ValueError):
        C.distill_loss(z.double(), t, i)
    with pytest.raises(ValueError):
        C.distill_loss(z, t, i[0])


def test_launch_choices(tmp_path):
    exe = str(tmp_path / "ffn_plan_sweep")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-include", "cmath", os.path.join(ROOT, "tests", "host", "ffn_plan_sweep.cpp"), "-o", exe],
                   check=True, capture_output=True, text=True)
    res = subprocess.run([exe, "3000"], capture_output=True, text=True)
    assert res.returncode == 0 and " 0 failures" in res.stdout, res.stdout + res.stderr


def test_kernels_do_not_spill(C, tmp_path):
    """No kernel of any device image in the library keeps vector registers in scratch memory."""
    llvm = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin")
    fat = str(tmp_path / "fat")
    if not os.path.exists(f"{llvm}/llvm-objcopy"):
        pytest.skip("llvm tools not installed")
    subprocess.run([f"{llvm}/llvm-objcopy", f"--dump-section=.hip_fatbin={fat}", C.LIB_PATH, str(tmp_path / "copy")],
                   check=True, capture_output=True)
    data = open(fat, "rb").read()
    names = []
    for i, at in enumerate(m.start() for m in re.finditer(b"__CLANG_OFFLOAD_BUNDLE__", data)):
        part, obj = str(tmp_path / f"part{i}"), str(tmp_path / f"obj{i}")
        open(part, "wb").write(data[at:])
        subprocess.run([f"{llvm}/clang-offload-bundler", "--type=o", "--unbundle", f"--input={part}",
                        f"--output={obj}", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950"], check=True, capture_output=True)
        notes = subprocess.run([f"{llvm}/llvm-readelf", "--notes", obj], check=True, capture_output=True, text=True).stdout
        for sym, spill in re.findall(r"\.symbol:\s+(\S+)[\s\S]*?\.vgpr_spill_count:\s+(\d+)", notes):
            names.append(sym)
            assert spill == "0", sym
    assert any("k_ffn" in n for n in names) and any("k_distill" in n for n in names)
