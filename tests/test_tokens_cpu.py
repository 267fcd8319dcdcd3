"""The paged 4-bit cache on the host: its layout, its bounds checks and its
refusals, compiled for the CPU."""

from __future__ import annotations

import os
import subprocess

from paper_2606_30709_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))


def test_layout_bounds_and_refusals(tmp_path):
    exe = str(tmp_path / "tokens_check")
    subprocess.run([build.HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", "-w",
                    "-I", build.INCLUDE, "-I", build.CSRC, os.path.join(HERE, "tokens_check.cpp"),
                    "-o", exe], check=True)
    r = subprocess.run([exe], stdout=subprocess.PIPE, text=True, timeout=60)
    assert r.returncode == 0, r.stdout
