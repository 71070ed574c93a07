"""The size of a plan's scratch where no device can be asked: an error, not a size that is kept for later calls."""
from __future__ import annotations

import os
import subprocess
import sys

from paper_2606_20855_gb300 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = """
from paper_2606_20855_gb300 import _abi, routing
for _ in range(2):
    for f in (lambda: _abi.ws_routing_scratch(2000, 8), lambda: routing._scratch(2000, 8, 0)):
        try:
            f()
        except _abi.WsError as e:
            assert e.status_name == "WS_ERR_CUDA" and "device query" in str(e), e
        else:
            raise SystemExit("a size without a device")
assert routing._scratch.cache_info().currsize == 0
"""


def test_no_device():
    build.build()
    res = subprocess.run([sys.executable, "-c", CODE], cwd=ROOT, env={**os.environ, "CUDA_VISIBLE_DEVICES": ""}, capture_output=True,
                         text=True, timeout=300)
    assert res.returncode == 0, res.stdout + res.stderr
