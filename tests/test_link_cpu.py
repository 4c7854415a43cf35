"""The library does not link without one of its kernels' objects (CPU only)."""

import os
import subprocess

import pytest

from paper_2609_21137_amd import build


def test_launchers_are_required(tmp_path, monkeypatch):
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not installed")
    monkeypatch.setattr(build, "BUILD", str(tmp_path))
    api = build._compile("cardan_api.hip")
    symbols = subprocess.run(["nm", "-C", api], check=True, capture_output=True, text=True).stdout.splitlines()
    for name in ("launch_ffn_forward", "launch_ffn_backward", "launch_distill", "launch_expert"):
        kinds = {line.split("cardan::")[0].split()[-1] for line in symbols if f"cardan::{name}(" in line}
        assert kinds == {"U"}, (name, kinds)
