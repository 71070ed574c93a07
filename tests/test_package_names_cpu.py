"""The package's name ``spgemm``: the submodule, which can be called like its function, in whatever order names are imported."""
from __future__ import annotations

import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = "paper_2606_20855_gb300"


@pytest.mark.parametrize("code", [
    f"from {P}.spgemm import DeviceCSR\nimport {P} as p\np.SpGEMM\nassert p.spgemm.SpGEMM is p.SpGEMM and callable(p.spgemm.spgemm)",
    f"import {P} as p\np.topk_route, p.DeviceCSR\nimport {P}.spgemm as m\nassert m.SpGEMM is p.SpGEMM",
    f"from {P} import spgemm\nimport {P}.spgemm\nassert callable(spgemm) and spgemm.DeviceCSR is {P}.spgemm.DeviceCSR",
    f"import {P}.spgemm\nfrom {P} import spgemm, Routing\nassert callable(spgemm) and {P}.spgemm.ewise is {P}.ewise",
    f"import {P}.routing\nimport {P} as p\nassert callable(p.spgemm) and p.spgemm.spmspv is p.spmspv",
])
def test_both_meanings_in_any_order(code):
    res = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stderr[-500:]


def test_call_of_the_module_is_one_of_the_function(monkeypatch):
    import paper_2606_20855_gb300 as p
    seen = []
    monkeypatch.setattr(p.spgemm, "spgemm", lambda *a, **k: seen.append((a, k)) or "C")
    assert p.spgemm("A", "B", validate=True) == "C" and seen == [(("A", "B"), {"validate": True})]
