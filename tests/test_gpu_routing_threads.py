"""Routing matrices from several threads at once."""
from __future__ import annotations

import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_plans_of_several_threads():
    """Plans of different sizes, built by threads on streams of their own."""
    from paper_2606_20855_gb300 import DeviceCSR, Routing
    failed = []

    def matrix(T, E, k):
        col = torch.rand((T, E), device="cuda").argsort(1)[:, :k].sort(1).values.to(torch.int32).flatten()
        return DeviceCSR(T, E, torch.arange(T + 1, device="cuda") * k, col, torch.ones(T * k, device="cuda"))

    def work(R):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                first = None
                for _ in range(300):
                    plan = Routing(R)
                    if first is None:
                        first = plan
                s.synchronize()
                assert torch.equal(plan.slots, first.slots) and torch.equal(plan.offsets, first.offsets)
                s.synchronize()
        except Exception as e:  # noqa: BLE001
            failed.append(e)

    sizes = [(1024, 1024, 4), (300, 1024, 2), (3000, 1024, 2), (3000, 900, 2)]
    mats = [matrix(*n) for n in sizes]
    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(R,)) for R in mats]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed, failed
