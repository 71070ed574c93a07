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


# Many tokens: v h is kept as a pair of 16-bit values, off by 2^-16 of it (bfloat16); in half by 2^-23 of it and, where the largest of
# 32 ranks of a token is brought to 1 or more, by 2^-25 of that largest one.
def _pairs(x, A, B, on, vals, dt):
    if dt == torch.bfloat16:
        return None
    extra = torch.zeros((x.shape[0], B.shape[1]), dtype=torch.float64, device="cuda")
    for a in range(on.shape[1]):
        t = on[:, a]
        vh = (vals[t, a].float().double()[:, None] * (x[t].double() @ A[a].double().T)).abs()
        for r0 in range(0, A.shape[1], 32):
            largest = vh[:, r0:r0 + 32].max(1, keepdim=True).values
            extra[t] += 2.0 ** -25 * largest * B[a][:, r0:r0 + 32].double().abs().sum(1)[None, :]
    return extra


def _check_tiles(x, A, B, on, vals, base):
    from paper_2606_20855_gb300 import adapters
    dt, K, r = x.dtype, x.shape[1], A.shape[1]
    got = adapters(x, A, B, _csr(on, vals), base, wait=True)
    want, mass = _exact(x, A, B, on, vals, base)
    bound = U[dt] * want.abs() + (K + 2 * r + 8) * 2.0 ** -23 * mass + STEP[dt]
    extra = _pairs(x, A, B, on, vals, dt)
    bound += 2.0 ** -16 * mass if extra is None else extra + 2.0 ** -23 * mass
    bad = ~((got.double() - want).abs() <= bound)
    if dt == torch.float16:  # from 65520 on a half is infinite
        bad &= ~(torch.isinf(got) & (want.abs() + bound >= 65520) & (got.sign() == want.sign()))
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4], want[bad][:4])


@pytest.mark.parametrize("size", [1e6, 2e5, 1.0, 1e-3, 1e-6, 1e-9])
@pytest.mark.parametrize("how", ["one", "runs", "several"])
@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("T,L,r,K,N", [(700, 5, 16, 64, 48), (300, 4, 40, 200, 300), (530, 3, 64, 72, 257), (600, 6, 13, 1000, 100)])
def test_many_tokens(T, L, r, K, N, dt, how, size):
    _check_tiles(*_case(T, L, r, K, N, dt, size, how))


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("r", [16, 48])
def test_values_far_apart(dt, r):
    """Adapters of one token, tokens of one tile and ranks of one adapter whose sizes differ by many powers of ten."""
    T, L, K, N = 600, 5, 96, 130
    x, A, B, on, vals, base = _case(T, L, r, K, N, dt, 1.0, "several")
    g = torch.Generator(device="cuda").manual_seed(7)
    vals = 10.0 ** (torch.rand((T, L), generator=g, device="cuda") * 10 - 7)
    _check_tiles(x, A, B, on, vals, base)
    ranks = 10.0 ** (torch.rand((1, r, 1), generator=g, device="cuda") * 7 - 5)
    _check_tiles(x, (A.float() * ranks).to(dt), B, on, vals, base)
    vals[::3] = 0.0  # entries that add nothing
    _check_tiles(x, A, B, on, vals, base)


@pytest.mark.parametrize("size", [1.0, 2e5, 1e-6])
def test_a_token_does_not_depend_on_its_tile(size):
    """Equal bits, whether all tokens of a tile share an adapter or every other one has another or none."""
    from paper_2606_20855_gb300 import adapters
    x, A, B, on, vals, base = _case(640, 4, 16, 128, 96, torch.float16, size, "one")
    all_one = adapters(x, A, B, _csr(on, vals), base)
    mixed = on.clone()
    mixed[1::4], mixed[2::4, 1], mixed[2::4, 3] = False, False, True
    some = adapters(x, A, B, _csr(mixed, vals), base)
    same = (mixed == on).all(1)
    assert bool(torch.isfinite(all_one).all()) and torch.equal(some[same], all_one[same])


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("r", [1, 15, 16, 40])
@pytest.mark.parametrize("T", [9, 700])
def test_infinite_sums_keep_their_sign(T, r, dt):
    """Positive matrices and one infinite value in x: infinity, not NaN, whatever the rank is padded to."""
    from paper_2606_20855_gb300 import adapters
    K, N = 72, 50
    x, A, B = _randn((T, K), dt, 1), _randn((2, r, K), dt, 2).abs() + 0.5, _randn((2, N, r), dt, 3).abs() + 0.5
    x[5, 3], x[8, 70] = float("inf"), -float("inf")
    on = torch.zeros((T, 2), dtype=torch.bool, device="cuda")
    on[:, 0], on[:, 1] = torch.arange(T, device="cuda") % 3 != 0, torch.arange(T, device="cuda") % 3 == 0
    on[5], on[8] = torch.tensor([False, True], device="cuda"), torch.tensor([False, True], device="cuda")
    y = adapters(x, A, B, _csr(on, torch.ones((T, 2), device="cuda")), None)
    assert bool((y[5] == float("inf")).all()) and bool((y[8] == -float("inf")).all())
    rest = torch.ones(T, dtype=torch.bool, device="cuda")
    rest[5], rest[8] = False, False
    assert bool(torch.isfinite(y[rest]).all())


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("r", [1, 15, 16, 40])
@pytest.mark.parametrize("T", [9, 700])
def test_infinite_sums_keep_their_sign_where_all_share_an_adapter(T, r, dt):
    """The same in tiles whose tokens have one adapter, none of which is computed by itself."""
    from paper_2606_20855_gb300 import adapters
    K, N = 72, 50
    x, A, B = _randn((T, K), dt, 1), _randn((1, r, K), dt, 2).abs() + 0.5, _randn((1, N, r), dt, 3).abs() + 0.5
    x[5, 3], x[8, 70] = float("inf"), -float("inf")
    y = adapters(x, A, B, _csr(torch.ones((T, 1), dtype=torch.bool, device="cuda"), torch.ones((T, 1), device="cuda")), None)
    assert bool((y[5] == float("inf")).all()) and bool((y[8] == -float("inf")).all())
    rest = torch.ones(T, dtype=torch.bool, device="cuda")
    rest[5], rest[8] = False, False
    assert bool(torch.isfinite(y[rest]).all())
