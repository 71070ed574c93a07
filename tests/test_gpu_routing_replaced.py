"""A routing matrix whose fields are replaced after its plan was built."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu


def _setup(T=300, E=12, k=3, H=64):
    from paper_2606_20855_gb300 import Routing, topk_route
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    R = topk_route(torch.randn((T, E), generator=g, device="cuda"), k)
    ys, gy = torch.randn((T * k, H), generator=g, device="cuda"), torch.randn((T, H), generator=g, device="cuda")
    return R, Routing(R), ys, gy


def _refill(*freed_bytes):
    """Takes the memory that was given back and fills it with NaN."""
    return [torch.full((n // 4,), float("nan"), device="cuda") for n in freed_bytes for _ in range(8)]


def test_values_replaced():
    """Weights rescaled into a new tensor, the old one's memory in other use."""
    R, plan, ys, gy = _setup()
    y, (gys, gvals) = plan.combine(ys), plan.combine_backward(gy, ys)
    n = R.vals.numel() * 4
    R.vals = R.vals * 2  # exact
    keep = _refill(n)
    assert torch.equal(plan.combine(ys), 2 * y)
    again = plan.combine_backward(gy, ys)
    assert torch.equal(again[0], 2 * gys) and torch.equal(again[1], gvals)
    del keep


def test_pattern_and_shape_replaced():
    """The plan is that of the matrix as it was built."""
    R, plan, ys, gy = _setup()
    y, x, offsets = plan.combine(ys), plan.dispatch(gy), plan.offsets.clone()
    n = R.colidx.numel() * 4
    R.rowptr, R.colidx = torch.zeros(301, dtype=torch.int64, device="cuda"), torch.zeros_like(R.colidx)
    R.nrows, R.ncols = 7, 2
    keep = _refill(n, 301 * 8)
    assert torch.equal(plan.combine(ys), y) and torch.equal(plan.dispatch(gy), x) and torch.equal(plan.offsets, offsets)
    W = torch.ones((12, 8, 64), dtype=torch.bfloat16, device="cuda")
    assert plan.matmul(ys.bfloat16(), W).shape == (900, 8)
    plan.wait()
    del keep


def test_values_that_do_not_fit_are_refused():
    R, plan, ys, gy = _setup()
    good = R.vals
    for vals, error in ((good.double(), TypeError), (good.cpu(), TypeError), (good[:-1], ValueError),
                        (torch.empty(2 * good.numel(), device="cuda")[::2], TypeError)):
        R.vals = vals
        with pytest.raises(error):
            plan.combine(ys)
        with pytest.raises(error):
            plan.combine_backward(gy, ys)
    R.vals = good
    plan.combine(ys)


def test_used_on_another_stream():
    """The values that a call on another stream reads stay allocated until it is done."""
    R, plan, ys, _ = _setup()
    want = plan.combine(ys)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    R.vals = R.vals.clone()
    s.wait_stream(torch.cuda.current_stream())
    got = plan.combine(ys, stream=s)
    R.vals = R.vals.clone()
    keep = _refill(R.vals.numel() * 4)
    s.synchronize()
    assert torch.equal(got, want)
    del keep
