"""The refusals of the routing, rows and optimizer calls under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only): the C ABI's host code is built with the
sanitizers and stand-ins for the kernels, as in tests/test_host_sanitizers.py, and
tests/test_rows_abi_cpu.py runs against it in a child process."""

import os
import subprocess
import sys

import pytest
from test_host_sanitizers import CLANGXX, CSRC, HIPCC, HOST, ROCM, ROOT, _asan_runtime, _run


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
def test_refusals_under_sanitizers(tmp_path):
    rt = _asan_runtime()
    if rt is None:
        pytest.skip("clang AddressSanitizer runtime not found")
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=all", "-Xarch_host", "-fno-omit-frame-pointer"]
    inc = ["-I", os.path.join(ROOT, "include")]
    api = str(tmp_path / "api.o")
    _run([HIPCC, "-O1", "-g", "-std=c++17", "-fPIC", "--offload-arch=gfx950", *san, *inc, "-c",
          os.path.join(CSRC, "cardan_api.hip"), "-o", api])
    host = ["-x", "c++", "-O1", "-g", "-std=c++17", "-fPIC", "-fsanitize=address,undefined",
            "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROCM, "include"), *inc]
    objs = [api]
    for src in (os.path.join(CSRC, "cardan_planner.cpp"), os.path.join(HOST, "kernel_stubs.cpp")):
        obj = str(tmp_path / (os.path.basename(src) + ".o"))
        _run([CLANGXX, *host, "-c", src, "-o", obj])
        objs.append(obj)
    lib = str(tmp_path / "libcardan_asan.so")
    _run([HIPCC, "-shared", "-fPIC", "--offload-arch=gfx950", "-Xarch_host", "-fsanitize=address",
          "-Xarch_host", "-fsanitize=undefined", "-shared-libsan", *objs, "-o", lib])
    env = {**os.environ, "CARDAN_LIB": lib, "LD_PRELOAD": rt,
           "ASAN_OPTIONS": "detect_leaks=0:halt_on_error=1", "UBSAN_OPTIONS": "halt_on_error=1:print_stacktrace=1"}
    res = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider",
                          os.path.join(ROOT, "tests", "test_rows_abi_cpu.py")],
                         capture_output=True, text=True, env=env, cwd=ROOT)
    out = res.stdout + res.stderr
    assert res.returncode == 0, out[-6000:]
    assert " passed" in res.stdout and " failed" not in res.stdout and " skipped" not in res.stdout, out[-3000:]
    assert "ERROR: AddressSanitizer" not in out and "runtime error:" not in out, out[-6000:]
