"""Operations on routing matrices where the dense matrices hold more than 2^32 values.

All but the last rows of an input are zero, and the last rows are compared with a 64-bit computation of them alone.  Bounds: a
value times a weight is rounded once (u |y|, u = 2^-8 for bfloat16), sums of n products of 32 bits add n 2^-23 of their mass.
"""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -8
LAST = 5


def _tail(rows, width, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    t = torch.zeros((rows, width), dtype=torch.bfloat16, device="cuda")
    t[-LAST:] = torch.randn((LAST, width), generator=g, device="cuda").bfloat16()
    return t


def _near(got, want, mass, terms):
    assert bool(((got.double() - want).abs() <= U * want.abs() + terms * 2.0 ** -23 * mass).all())


def test_rows_there_and_back():
    from paper_2606_20855_gb300 import DeviceCSR, Routing
    T, E, H = 70_001, 4, 32_768
    col = torch.tensor([1, 3], dtype=torch.int32, device="cuda").repeat(T)
    v = torch.rand(2 * T, device="cuda") + 0.5
    plan = Routing(DeviceCSR(T, E, torch.arange(T + 1, device="cuda") * 2, col, v))
    x = _tail(T, H, 1)
    xs = plan.dispatch(x)
    assert xs.numel() > 2 ** 32
    assert torch.equal(xs[T - LAST:T], x[-LAST:]) and torch.equal(xs[-LAST:], x[-LAST:])
    assert not bool(xs[:2].any()) and not bool(xs[T:T + 2].any())
    last, w = x[-LAST:].double(), v.view(T, 2)[-LAST:].double()
    y = plan.combine(xs)
    _near(y[-LAST:], last * w.sum(1, keepdim=True), last.abs() * w.sum(1, keepdim=True), 2)
    gys, gv = plan.combine_backward(x, xs)
    _near(gys[-LAST:], last * w[:, 1:], last.abs() * w[:, 1:], 1)
    dot = (last * last).sum(1, keepdim=True)
    assert bool(((gv.view(T, 2)[-LAST:].double() - dot).abs() <= H * 2.0 ** -23 * dot).all())
    gx = plan.dispatch_backward(gys)
    both = (gys[T - LAST:T].double() + gys[-LAST:].double())
    _near(gx[-LAST:], both, both.abs(), 2)


def test_products():
    from paper_2606_20855_gb300 import DeviceCSR, Routing
    T, K, N = 2_200_001, 64, 2048
    col = (torch.arange(T, device="cuda") % 2).to(torch.int32)
    plan = Routing(DeviceCSR(T, 2, torch.arange(T + 1, device="cuda"), col, torch.ones(T, device="cuda")))
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    W = torch.randn((2, N, K), generator=g, device="cuda").bfloat16()
    xs, gys = _tail(T, K, 3), _tail(T, N, 4)
    ys = plan.matmul(xs, W)
    assert ys.numel() > 2 ** 32
    a, b, w = xs[-LAST:].double(), gys[-LAST:].double(), W[1].double()
    _near(ys[-LAST:], a @ w.T, a.abs() @ w.abs().T, K)
    gxs, gW = plan.matmul_backward(gys, xs, W)
    _near(gxs[-LAST:], b @ w, b.abs() @ w.abs(), N)
    _near(gW[1], b.T @ a, b.abs().T @ a.abs(), LAST)
    assert not bool(gW[0].any()) and not bool(gxs[:-LAST].any())


def test_adapters():
    from paper_2606_20855_gb300 import DeviceCSR, adapters
    T, K, N, L, r = 2_200_001, 64, 2048, 3, 16
    col = (torch.arange(T, device="cuda") % L).to(torch.int32)
    S = DeviceCSR(T, L, torch.arange(T + 1, device="cuda"), col, torch.full((T,), 0.5, device="cuda"))
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    A = torch.randn((L, r, K), generator=g, device="cuda").bfloat16()
    B = torch.randn((L, N, r), generator=g, device="cuda").bfloat16()
    x, base = _tail(T, K, 6), _tail(T, N, 7)
    y = adapters(x, A, B, S, base, wait=True)
    assert y.numel() > 2 ** 32 and not bool(y[:3].any())
    for i in range(T - LAST, T):
        a, b, xi, bi = A[i % L].double(), B[i % L].double(), x[i].double(), base[i].double()
        want = bi + 0.5 * (b @ (a @ xi))
        mass = bi.abs() + 0.5 * (b.abs() @ (a.abs() @ xi.abs()))
        # the inner products are kept as pairs of bfloat16: 2^-16 of them
        assert bool(((y[i].double() - want).abs() <= U * want.abs() + ((K + 2 * r + 8) * 2.0 ** -23 + 2.0 ** -16) * mass).all())
