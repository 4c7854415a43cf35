"""Launch choices of the feed-forward block count the workgroups that a CU holds (CPU only)."""

import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_workgroups_of_a_cu(tmp_path):
    exe = str(tmp_path / "ffn_resident_sweep")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    os.path.join(ROOT, "tests", "host", "ffn_resident_sweep.cpp"), "-o", exe],
                   check=True, capture_output=True, text=True)
    res = subprocess.run([exe], capture_output=True, text=True)
    assert res.returncode == 0 and res.stdout.startswith("0 failures"), res.stdout + res.stderr
