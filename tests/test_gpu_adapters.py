"""Low-rank adapters of many requests on the GPU against a 64-bit computation.

Tolerance.  With n = K inner products' terms, h is off by at most K 2^-23 sum |A x| (32-bit sums) and, kept as a pair of 16-bit
values, by 2^-16 |h| (bfloat16: 2^-8 of a remainder below 2^-8 |h|) or 2^-22 |h| + 2^-25 (half); the result's 32-bit sum of r
products an adapter adds r 2^-23 of their sum, the rounding u |y|.  So the bound is
u |y| + (K + 2 r + 8) 2^-23 mass + pair * mass, mass = |base| + |v| |B| |A| |x|.
"""
from __future__ import annotations

import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
PAIR = {torch.bfloat16: 2.0 ** -16, torch.float16: 2.0 ** -21}
TYPES = [torch.bfloat16, torch.float16]


def _randn(shape, dt, seed, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dt)


def _select(T, L, how, seed):
    """S by a mask: "runs" of tokens with one adapter, "own" adapter each, "mixed" 0..3 of them, "none"."""
    from paper_2606_20855_gb300 import DeviceCSR
    g = torch.Generator().manual_seed(seed)
    on = torch.zeros((T, L), dtype=torch.bool)
    if how == "runs":
        of = torch.arange(T) // 50 * 7 % (L + 1)
        on[of < L, of[of < L]] = True
    elif how == "own":
        on[torch.arange(T), torch.randint(0, L, (T,), generator=g)] = True
    elif how == "mixed":
        on = torch.rand((T, L), generator=g) < min(1.0, 1.5 / L)
    rowptr = torch.zeros(T + 1, dtype=torch.int64)
    rowptr[1:] = torch.cumsum(on.sum(1), 0)
    col = on.nonzero()[:, 1].to(torch.int32).cuda()
    return DeviceCSR(T, L, rowptr.cuda(), col, _randn(col.numel(), torch.float32, seed + 1))


def _dense(S):
    D = torch.zeros((S.nrows, S.ncols), dtype=torch.float64, device="cuda")
    row = torch.repeat_interleave(torch.arange(S.nrows, device="cuda"), S.rowptr[1:] - S.rowptr[:-1])
    D[row, S.colidx.long()] = S.vals.double()
    return D


def _check(x, A, B, S, base, got):
    D, (L, r, K) = _dense(S), A.shape
    want = base.double() if base is not None else torch.zeros((x.shape[0], B.shape[1]), dtype=torch.float64, device="cuda")
    mass = want.abs()
    for a in range(L):
        t = D[:, a] != 0
        v, xa = D[t, a][:, None], x[t].double()
        want[t] += v * (xa @ A[a].double().T @ B[a].double().T)
        mass[t] += v.abs() * (xa.abs() @ A[a].double().abs().T @ B[a].double().abs().T)
    assert got.shape == want.shape and got.dtype == x.dtype
    dt = x.dtype
    bound = U[dt] * want.abs() + ((K + 2 * r + 8) * 2.0 ** -23 + PAIR[dt]) * mass + (1e-6 if dt == torch.float16 else 0.0)
    bad = (got.double() - want).abs() > bound
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4], want[bad][:4])


@pytest.mark.parametrize("T", [1, 2, 33, 129, 513, 700])
@pytest.mark.parametrize("L,r,K,N", [(1, 16, 64, 64), (5, 8, 40, 1000), (12, 4, 1001, 24), (40, 32, 512, 515), (3, 64, 264, 2048),
                                     (6, 1, 17, 9), (4, 13, 300, 72), (2, 100, 96, 130)])
@pytest.mark.parametrize("how", ["runs", "own", "mixed", "none"])
@pytest.mark.parametrize("dt", TYPES)
def test_against_64_bits(T, L, r, K, N, how, dt):
    from paper_2606_20855_gb300 import adapters
    x, A, B = _randn((T, K), dt, 1), _randn((L, r, K), dt, 2, K ** -0.5), _randn((L, N, r), dt, 3, r ** -0.5)
    S, base = _select(T, L, how, T + L), _randn((T, N), dt, 4)
    _check(x, A, B, S, base, adapters(x, A, B, S, base))
    _check(x, A, B, S, None, adapters(x, A, B, S))


@pytest.mark.parametrize("T", [20, 300, 600])
def test_strides_alignment_and_in_place(T):
    from paper_2606_20855_gb300 import adapters
    L, r, K, N = 4, 16, 104, 120
    for dt in TYPES:
        wx, wb = _randn((T, 200), dt, 1), _randn((T, 260), dt, 2)
        WA, WB = _randn((L, r, 160), dt, 3, 0.1), _randn((L, N, 40), dt, 4, 0.3)
        S = _select(T, L, "mixed", T)
        for skip in (0, 1, 2, 4, 8):
            x, A, B, base = wx[:, skip:skip + K], WA[:, :, skip:skip + K], WB[:, :, skip:skip + r], wb[:, skip:skip + N]
            y = adapters(x, A, B, S, base)
            _check(x, A, B, S, base, y)
            assert torch.equal(y, adapters(x, A, B, S, base.contiguous()))
            buf = wb.clone()
            part = buf[:, skip:skip + N]
            assert adapters(x, A, B, S, part, out=part) is part
            assert torch.equal(part, y)
            buf[:, skip:skip + N] = wb[:, skip:skip + N]
            assert torch.equal(buf, wb)  # nothing else was written
        t = _randn((K, T), dt, 5).t()
        _check(t, WA[:, :, :K], WB.transpose(1, 2)[:, :N].transpose(1, 2)[:, :, :r], S, None,
               adapters(t, WA[:, :, :K], WB[:, :, :r], S))


@pytest.mark.parametrize("T", [40, 200, 600])
def test_infinities_stay_with_their_tokens(T):
    from paper_2606_20855_gb300 import adapters
    L, r, K, N = 6, 8, 64, 96
    x, A, B = _randn((T, K), torch.bfloat16, 1), _randn((L, r, K), torch.bfloat16, 2), _randn((L, N, r), torch.bfloat16, 3)
    S, base = _select(T, L, "own", 5), _randn((T, N), torch.bfloat16, 4)
    A[1], B[2], x[7] = math.nan, math.inf, math.inf
    D = _dense(S) != 0
    y = adapters(x, A, B, S, base)
    hit = D[:, 1] | D[:, 2]
    hit[7] = True
    assert torch.equal(~torch.isfinite(y).all(1), hit)


def test_columns_out_of_range_take_no_part():
    from paper_2606_20855_gb300 import DeviceCSR, adapters
    for T in (8, 256, 600):
        x, A, B = _randn((T, 32), torch.float16, 1), _randn((3, 8, 32), torch.float16, 2), _randn((3, 16, 8), torch.float16, 3)
        col = torch.ones(T, dtype=torch.int32, device="cuda")
        col[2], col[3] = -7, 3
        rowptr = torch.arange(T + 1, device="cuda")
        y = adapters(x, A, B, DeviceCSR(T, 3, rowptr, col, torch.ones(T, device="cuda")))
        assert bool((y[2:4] == 0).all()) and bool((y[:2] != 0).any(1).all()) and bool((y[4:] != 0).any(1).all())


def test_empty_sizes():
    from paper_2606_20855_gb300 import adapters
    bf = torch.bfloat16
    for T, L, r, K, N in ((0, 3, 8, 16, 8), (5, 3, 0, 16, 8), (5, 3, 8, 0, 8), (5, 3, 8, 16, 0), (300, 3, 8, 0, 8), (600, 3, 8, 0, 8), (600, 3, 0, 8, 8)):
        base = _randn((T, N), bf, 0)
        y = adapters(_randn((T, K), bf, 1), _randn((L, r, K), bf, 2), _randn((L, N, r), bf, 3), _select(T, L, "own", 1), base)
        assert torch.equal(y, base)


def test_beside_the_shared_projection():
    """The projection of all tokens is a product with one expert; its result is the adapters' base."""
    from paper_2606_20855_gb300 import DeviceCSR, Routing, adapters
    T, L, r, K, N = 150, 4, 16, 128, 192
    x, W = _randn((T, K), torch.bfloat16, 1), _randn((1, N, K), torch.bfloat16, 2, K ** -0.5)
    A, B = _randn((L, r, K), torch.bfloat16, 3, K ** -0.5), _randn((L, N, r), torch.bfloat16, 4, r ** -0.5)
    one = DeviceCSR(T, 1, torch.arange(T + 1, device="cuda"), torch.zeros(T, dtype=torch.int32, device="cuda"), torch.ones(T, device="cuda"))
    base = Routing(one).matmul(x, W)
    S = _select(T, L, "runs", 1)
    want = base.clone()
    _check(x, A, B, S, want, adapters(x, A, B, S, base, out=base))


@pytest.mark.parametrize("how", ["none", "runs"])
def test_base_from_the_product_before(how):
    """base is the result of a product that may still run when the call is queued."""
    from paper_2606_20855_gb300 import DeviceCSR, Routing, adapters
    T, K, N, L, r, dt = 4096, 1024, 1024, 4, 16, torch.bfloat16
    x, W = _randn((T, K), dt, 90), _randn((1, N, K), dt, 91, K ** -0.5)
    A, B = _randn((L, r, K), dt, 92, K ** -0.5), _randn((L, N, r), dt, 93)
    one = DeviceCSR(T, 1, torch.arange(T + 1, device="cuda"), torch.zeros(T, dtype=torch.int32, device="cuda"),
                    torch.ones(T, device="cuda"))
    plan, S = Routing(one), _select(T, L, how, 94)
    torch.cuda.synchronize()
    for _ in range(4):
        base = plan.matmul(x, W)
        got = adapters(x, A, B, S, base, wait=True)
        _check(x, A, B, S, base, got)
        base.fill_(float("nan"))


def test_equal_inputs_give_equal_bits():
    from paper_2606_20855_gb300 import adapters
    for T in (30, 900):
        args = (_randn((T, 512), torch.bfloat16, 1), _randn((9, 16, 512), torch.bfloat16, 2), _randn((9, 300, 16), torch.bfloat16, 3),
                _select(T, 9, "mixed", 2), _randn((T, 300), torch.bfloat16, 4))
        assert torch.equal(adapters(*args), adapters(*args))


def test_refusals():
    from paper_2606_20855_gb300 import DeviceCSR, adapters
    x, A, B = _randn((4, 16), torch.float16, 1), _randn((3, 8, 16), torch.float16, 2), _randn((3, 24, 8), torch.float16, 3)
    S = _select(4, 3, "own", 1)
    with pytest.raises(ValueError):
        adapters(x[:3], A, B, S)
    with pytest.raises(ValueError):
        adapters(x, A[:2], B, S)
    with pytest.raises(ValueError):
        adapters(x, A, B[:, :, :4], S)
    with pytest.raises(ValueError):
        adapters(x[:, :8], A, B, S)
    with pytest.raises(ValueError):
        adapters(x, A, B, S, torch.zeros((4, 23), dtype=torch.float16, device="cuda"))
    with pytest.raises(ValueError):
        adapters(x, A[:2], B[:2], S)
    with pytest.raises(TypeError):
        adapters(x, A.float(), B, S)
    with pytest.raises(TypeError):
        adapters(x, A, B, S, torch.zeros((4, 24), device="cuda"))
    with pytest.raises(TypeError):
        adapters(x, A, B, DeviceCSR(4, 3, S.rowptr, S.colidx, S.vals.double()))
    from paper_2606_20855_gb300 import _abi
    with pytest.raises(_abi.WsError) as e:
        adapters(x.float(), A.float(), B.float(), S)
    assert e.value.status_name == "WS_ERR_DTYPE"
    big = torch.zeros((8, 24), dtype=torch.float16, device="cuda")
    with pytest.raises(ValueError):
        adapters(x, A, B, S, big[:4], out=big[1:5])
