"""Launches of a routing matrix's plan on a fake CUDA runtime (no GPU): plans built by several threads."""
from __future__ import annotations

import os
import subprocess

from paper_2606_20855_gb300 import build

HERE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "host_runtime")


def test_plans_of_several_threads(tmp_path):
    exe = str(tmp_path / "plan_checks")
    srcs = [os.path.join(build.CSRC, "routing.cu"), os.path.join(HERE, "plan_checks.cpp")]
    res = subprocess.run([build.nvcc(), *build.ARCH, "-O1", "-std=c++17", "--expt-relaxed-constexpr", "-cudart", "none", "-I", build.INCLUDE,
                          "-I", build.CSRC, *srcs, "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stdout + res.stderr
    res = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert res.returncode == 0, res.stdout + res.stderr
