"""The library does not link without the routing's, the rows' and the optimizer's objects (CPU only)."""

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
    for name in ("launch_route", "launch_route_backward", "launch_dispatch", "launch_combine", "launch_combine_backward",
                 "launch_adamw"):
        kinds = {line.split("cardan::")[0].split()[-1] for line in symbols if f"cardan::{name}(" in line}
        assert kinds == {"U"}, (name, kinds)
