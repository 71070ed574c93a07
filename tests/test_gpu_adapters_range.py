"""Adapters whose inner products, times S's values, are large or small beside what 16-bit values hold.

Tolerance.  A result is a sum in 32 bits of base and of r products an adapter, each of B and a 32-bit sum of K products times the
value: off by at most u |y| + (K + 2 r + 8) 2^-23 mass with mass = |base| + |v| |B| |A| |x|, and half a step of the result's type
near zero.  Few tokens: nothing else is rounded.
"""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
STEP = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}  # half the smallest step
TYPES = [torch.bfloat16, torch.float16]


def _randn(shape, dt, seed, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dt)


def _csr(on, vals):
    """S from a mask and a value of every place."""
    from paper_2606_20855_gb300 import DeviceCSR
    rowptr = torch.zeros(on.shape[0] + 1, dtype=torch.int64, device="cuda")
    rowptr[1:] = torch.cumsum(on.sum(1), 0)
    return DeviceCSR(on.shape[0], on.shape[1], rowptr, on.nonzero()[:, 1].to(torch.int32), vals[on].float().contiguous())


def _exact(x, A, B, on, vals, base):
    want, mass = base.double(), base.double().abs()
    for a in range(on.shape[1]):
        t = on[:, a]
        v, xa = vals[t, a].float().double()[:, None], x[t].double()
        want[t] += v * (xa @ A[a].double().T @ B[a].double().T)
        mass[t] += v.abs() * (xa.abs() @ A[a].double().abs().T @ B[a].double().abs().T)
    return want, mass


def _case(T, L, r, K, N, dt, size, how):
    """v h of about `size`, B so that the result is about one."""
    x, A = _randn((T, K), dt, 1), _randn((L, r, K), dt, 2, K ** -0.5)
    B, base = (_randn((L, N, r), torch.float32, 3).clamp(-4, 4) * min(1e4, r ** -0.5 / size)).to(dt), _randn((T, N), dt, 4)
    t = torch.arange(T, device="cuda")
    on = torch.zeros((T, L), dtype=torch.bool, device="cuda")
    if how == "one":  # all tokens share an adapter
        on[:, 1 % L] = True
    elif how == "runs":  # some have none
        of = t // 50 * 7 % (L + 1)
        on[of < L, of[of < L]] = True
    else:  # several each
        on = torch.rand((T, L), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda") < 0.6
    vals = (_randn((T, L), torch.float32, 6).abs() + 0.5) * size
    return x, A, B, on, vals, base


@pytest.mark.parametrize("size", [1e6, 2e5, 1.0, 1e-3, 1e-6, 1e-9])
@pytest.mark.parametrize("how", ["one", "runs", "several"])
@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("T,L,r,K,N", [(1, 2, 16, 64, 48), (40, 4, 13, 200, 100)])
def test_few_tokens(T, L, r, K, N, dt, how, size):
    from paper_2606_20855_gb300 import adapters
    x, A, B, on, vals, base = _case(T, L, r, K, N, dt, size, how)
    got = adapters(x, A, B, _csr(on, vals), base)
    want, mass = _exact(x, A, B, on, vals, base)
    bound = U[dt] * want.abs() + (K + 2 * r + 8) * 2.0 ** -23 * mass + STEP[dt]
    bad = ~((got.double() - want).abs() <= bound)
    assert not bool(bad.any()), (int(bad.sum()), got[bad][:4], want[bad][:4])
