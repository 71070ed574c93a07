"""The package's public names, imported the ways a program imports them, each in a process of its own."""
from __future__ import annotations

import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("code", [
    "from paper_2606_20855_gb300 import DeviceCSR, SpGEMM, spgemm; assert callable(spgemm)",
    "from paper_2606_20855_gb300 import *; assert callable(spgemm) and callable(topk_route)",
    "from paper_2606_20855_gb300 import Routing; from paper_2606_20855_gb300.spgemm import SpGEMM, spgemm",
    "import paper_2606_20855_gb300 as p; assert callable(p.spgemm) and all(hasattr(p, n) for n in p.__all__)",
    "from paper_2606_20855_gb300.spgemm import spgemm; import paper_2606_20855_gb300 as p; p.SpGEMM",
    "import paper_2606_20855_gb300 as p; assert not hasattr(p, 'no_such_name')",
])
def test_public_names(code):
    res = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stderr[-500:]
