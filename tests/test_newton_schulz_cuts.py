"""The rule that cuts a Newton-Schulz step's products, against measured times (no GPU)."""

import os
import shutil
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_cuts_are_near_the_fastest_of_those_measured(tmp_path):
    gxx = shutil.which("g++")
    assert gxx, "g++ is part of the image"
    csrc, exe = os.path.join(ROOT, "paper_2605_21177_amd", "csrc"), str(tmp_path / "ns_cut_times")
    cmd = [gxx, "-std=c++17", "-O1", "-I", csrc, os.path.join(ROOT, "tests", "ns_cut_times.cpp"), os.path.join(csrc, "layers_shape.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout.startswith("ok:"), r.stdout
