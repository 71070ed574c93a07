"""Calls on tensors of another device than the current one (a fake answer for the current one) are refused before anything is queued."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_another_device_is_current(monkeypatch):
    from paper_2606_20855_gb300 import DeviceCSR, Routing, adapters, routing, topk_route, topk_route_backward
    bf = torch.bfloat16
    logits, x, W = torch.randn((20, 8), device="cuda"), torch.ones((20, 16), dtype=bf, device="cuda"), torch.ones((8, 16, 16), dtype=bf, device="cuda")
    R = topk_route(logits, 2)
    plan = Routing(R)
    xs, g = plan.dispatch(x), torch.ones(40, device="cuda")
    S = DeviceCSR(20, 1, torch.arange(21, device="cuda"), torch.zeros(20, dtype=torch.int32, device="cuda"), torch.ones(20, device="cuda"))
    A = torch.ones((1, 16, 16), dtype=bf, device="cuda")
    calls = [lambda: topk_route(logits, 2), lambda: topk_route_backward(logits, R, g), lambda: Routing(R), lambda: plan.dispatch(x),
             lambda: plan.dispatch_backward(xs), lambda: plan.combine(xs), lambda: plan.combine_backward(x, xs), lambda: plan.matmul(xs, W),
             lambda: plan.matmul_backward(xs, xs, W), lambda: plan.wait(), lambda: adapters(x, A, A, S)]
    with monkeypatch.context() as m:
        m.setattr(routing, "_current_device", lambda: x.device.index + 1)
        for f in calls:
            with pytest.raises(ValueError, match="current"):
                f()
    for f in calls:
        f()
    torch.cuda.synchronize()
