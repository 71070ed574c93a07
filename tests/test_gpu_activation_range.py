"""Activations and their derivatives at every finite value of both 16-bit types and at infinities, relative to the result.

Rows of no values make the bias the sum, and the sums given to the backward pass may be any: so both are seen alone.  Bounds, with e = 2^-23
for an operation in 32 bits and u half a step of the type:
  logistic function of v      the exponent is off by e |v| and 2^-23, power and reciprocal by 2^-22: relative (8 + 2 |v|) e
  normal distribution         the approximation of its tail by 3.1e-5 of it, six sums by 8 e, the exponent z^2 / 2 by e z^2: relative
                              3.3e-5 + e z^2; above 0 it is 1 less that tail
  a product or sum of them    its terms' bounds and e each
  what is below 2^-126 may be 0: the logistic function, multiplied by at most 88 in values and 235 in derivatives (gelu_tanh's argument has
                              a derivative of 23 at -10.1), and exp(-z^2 / 2), multiplied by at most 5.3: values to 2^-119, derivatives to
                              2^-118
"""
from __future__ import annotations

import math

import pytest
import torch

from tests._fused import E32, FLOOR, TYPES, U, plan_of

pytestmark = pytest.mark.gpu

TAILS = ["silu", "gelu", "gelu_tanh", "sigmoid"]


def every(dt):
    v = torch.arange(65536, dtype=torch.int32, device="cuda").to(torch.int16).view(dt)
    return v[torch.isfinite(v)]


def exact(act, z):
    """Value, derivative, and how far either may be off, in 64 bits, without differences of nearly equal numbers."""
    if act == "gelu":
        lower = 0.5 * torch.special.erfc(z.abs() / math.sqrt(2))  # 1 - Phi(|z|)
        dense = torch.exp(-z * z / 2) / math.sqrt(2 * math.pi) * z.abs()
        off = (3.3e-5 + E32 * z * z).clamp(max=1.0)
        phi = torch.where(z < 0, lower, 1 - lower)
        return (z * phi, torch.where(z < 0, lower - dense, 1 - lower + dense), z.abs() * (lower * off + 2 * E32 * phi),
                (lower + dense) * off + 4 * E32 * (phi + dense))
    v, dv = z, torch.ones_like(z)
    if act == "gelu_tanh":
        a = math.sqrt(8 / math.pi)
        v, dv = a * (z + 0.044715 * z ** 3), a * (1 + 0.134145 * z * z)
    s, other = torch.sigmoid(v), torch.sigmoid(-v)
    off = ((8 + 2 * v.abs()) * E32).clamp(max=1.0)
    # what is off by `off` is the exponential: the function itself by that times 1 - s above 0
    s_off = s * (off * other + 4 * E32)
    if act == "sigmoid":
        return s, s * other, s_off, s * other * (2 * off + 4 * E32)
    bend = z.abs() * dv * s * other
    return z * s, s + z * dv * s * other, z.abs() * s_off + E32 * z.abs() * s, s_off + bend * (2 * off + 8 * E32)


def near(got, want, off, dt, small):
    bound = U[dt] * want.abs() + (1 + U[dt]) * off + FLOOR[dt] + small
    bad = ~((got.double() - want).abs() <= bound)
    assert not bool(bad.any()), (int(bad.sum()), got[bad][:4].tolist(), want[bad][:4].tolist(), bound[bad][:4].tolist())


@pytest.mark.parametrize("rows", [2, 30, 200])
@pytest.mark.parametrize("act", TAILS)
@pytest.mark.parametrize("dt", TYPES)
def test_every_value(dt, act, rows):
    z = every(dt)
    plan, N = plan_of([rows]), z.numel()
    xs, W = torch.zeros((rows, 0), dtype=dt, device="cuda"), torch.zeros((1, N, 0), dtype=dt, device="cuda")
    ys, kept = plan.linear(xs, W, z[None], act, keep=True)
    assert torch.equal(kept, z.expand(rows, N)) and torch.equal(ys, ys[:1].expand(rows, N))
    h = plan.gated(xs, W, W, act, z[None], torch.ones((1, N), dtype=dt, device="cuda"))
    assert torch.equal(h, ys)
    value, slope, value_off, slope_off = exact(act, z.double())
    near(ys[0], value, value_off, dt, 2.0 ** -119)
    if rows == 2:  # one of the two rows alone has a gradient: the bias's is the derivative, in 32 bits until it is rounded
        g = torch.zeros((rows, N), dtype=dt, device="cuda")
        g[1] = 1
        _, _, gb = plan.linear_backward(g, xs, W, kept, act, bias=True)
        near(gb[0], slope, slope_off, dt, 2.0 ** -118)


@pytest.mark.parametrize("act", TAILS + ["relu"])
@pytest.mark.parametrize("rows", [2, 30, 200])
def test_limits(rows, act):
    """At infinities, and far from 0 on both sides, values and derivatives are the limits themselves."""
    dt = torch.bfloat16
    low = torch.tensor([-math.inf, -3e38, -1e30, -1e4, -200.0, -110.0], dtype=dt, device="cuda")
    plan, N = plan_of([rows]), 2 * low.numel()
    xs, W = torch.zeros((rows, 0), dtype=dt, device="cuda"), torch.zeros((1, N, 0), dtype=dt, device="cuda")
    z = torch.cat([low, -low])
    ys, kept = plan.linear(xs, W, z[None], act, keep=True)
    high = torch.ones_like(low) if act == "sigmoid" else -low
    assert not bool(ys[:, :low.numel()].any()) and torch.equal(ys[:, low.numel():], high.expand(rows, low.numel()))
    _, _, gb = plan.linear_backward(torch.ones_like(ys), xs, W, kept, act, bias=True)
    assert not bool(gb[0, :low.numel()].any())
    assert bool((gb[0, low.numel():] == (0 if act == "sigmoid" else rows)).all())
