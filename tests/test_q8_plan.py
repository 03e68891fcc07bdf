"""The 8-bit attention's launch plan, compiled for the host and run over random calls (q8_plan_check.cpp)."""

import os
import subprocess

from paper_2609_11582_amd import _build


def test_plan_covers_every_row_once_and_stays_in_the_workspace(tmp_path):
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "q8_plan_check.cpp")
    exe = str(tmp_path / "q8_plan_check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", _build.CSRC, src, "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout[-2000:] + r.stderr[-2000:]
