"""The experts' products (by column of a routing matrix) and their gradients on the GPU against 64-bit products.

Tolerance: a result is a sum of n products of 16-bit values, exact in 32 bits each, in a tree of 32-bit additions, rounded
once: off by at most u |y| + n 2^-23 sum |products| (tensor cores may truncate where they align addends, so a unit of
2^-23 for each addition).
"""
from __future__ import annotations

import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TYPES = [torch.bfloat16, torch.float16]


def _randn(shape, dt, seed, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dt)


def _plan(counts):
    """A plan whose column e has counts[e] entries, one entry a row."""
    from paper_2606_20855_gb300 import DeviceCSR, Routing
    E, Z = len(counts), sum(counts)
    col = torch.repeat_interleave(torch.arange(E), torch.tensor(counts))
    col = col[torch.randperm(Z, generator=torch.Generator().manual_seed(Z))].to(torch.int32).cuda()
    return Routing(DeviceCSR(Z, E, torch.arange(Z + 1, device="cuda"), col, torch.ones(Z, device="cuda")))


def _near(got, want, mass, n, dt):
    bound = U[dt] * want.abs() + n * 2.0 ** -23 * mass + (2.0 ** -24 if dt == torch.float16 else 0.0)
    bad = (got.double() - want).abs() > bound
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4], want[bad][:4])


def _check(plan, counts, xs, W, gys, grad=True):
    dt, (E, N, K) = xs.dtype, W.shape
    ys = plan.matmul(xs, W)
    gxs, gW = plan.matmul_backward(gys, xs, W) if grad else (None, None)
    plan.wait()
    assert ys.shape == (xs.shape[0], N) and ys.dtype == dt
    at = 0
    for e, n in enumerate(counts):
        x, g, w = xs[at:at + n].double(), gys[at:at + n].double(), W[e].double()
        _near(ys[at:at + n], x @ w.T, x.abs() @ w.abs().T, K, dt)
        if grad:
            _near(gxs[at:at + n], g @ w, g.abs() @ w.abs(), N, dt)
            _near(gW[e], g.T @ x, g.abs().T @ x.abs(), n, dt)
        at += n


COUNTS = {
    "one": [1],
    "first of two": [1, 0],
    "few": [0, 3, 0, 1, 16, 17, 0, 2],
    "tiles": [128, 64, 256, 0, 65],
    "ragged": [1, 127, 129, 0, 0, 300, 63, 64],
    "alone": [777],
    "many": [(7 * e) % 23 for e in range(150)],
    "lopsided": [0] * 20 + [1500] + [1] * 11,
}


@pytest.mark.parametrize("name", list(COUNTS))
@pytest.mark.parametrize("N,K", [(8, 8), (128, 64), (256, 320), (72, 1000), (1003, 40), (17, 9), (520, 136)])
@pytest.mark.parametrize("dt", TYPES)
def test_products_and_gradients(name, N, K, dt):
    counts = COUNTS[name]
    Z = sum(counts)
    _check(_plan(counts), counts, _randn((Z, K), dt, 1), _randn((len(counts), N, K), dt, 2, 0.3), _randn((Z, N), dt, 3))


def test_many_tiles_per_sm():
    """More tiles than SMs, so that every CTA goes through its stages and accumulators many times."""
    counts = [1000, 3, 2100, 640, 0, 911]
    Z = sum(counts)
    _check(_plan(counts), counts, _randn((Z, 712), torch.bfloat16, 1), _randn((6, 2056, 712), torch.bfloat16, 2, 0.3),
           _randn((Z, 2056), torch.bfloat16, 3))
    counts = [700, 0, 1300, 5, 2000]  # tiles in pairs, in all three products
    Z = sum(counts)
    _check(_plan(counts), counts, _randn((Z, 2304), torch.float16, 1), _randn((5, 1280, 2304), torch.float16, 2, 0.3),
           _randn((Z, 1280), torch.float16, 3))
    counts = [9] * 900
    _check(_plan(counts), counts, _randn((8100, 264), torch.float16, 1), _randn((900, 400, 264), torch.float16, 2, 0.3),
           _randn((8100, 400), torch.float16, 3))


def test_single_values():
    """One nonzero in each operand: every place of a result holds what its formula says, exactly."""
    counts = [70, 130, 5]
    plan, Z, N, K = _plan(counts), 205, 200, 150
    for row, n, k in ((0, 0, 0), (69, 199, 149), (70, 63, 64), (199, 128, 65), (204, 127, 17)):
        e = 0 if row < 70 else 1 if row < 200 else 2
        xs = torch.zeros((Z, K), dtype=torch.bfloat16, device="cuda")
        W = torch.zeros((3, N, K), dtype=torch.bfloat16, device="cuda")
        gys = torch.zeros((Z, N), dtype=torch.bfloat16, device="cuda")
        xs[row, k], W[e, n, k], gys[row, n] = 3.0, 5.0, 7.0
        ys = plan.matmul(xs, W)
        gxs, gW = plan.matmul_backward(gys, xs, W)
        for got, at, value in ((ys, (row, n), 15.0), (gxs, (row, k), 35.0), (gW, (e, n, k), 21.0)):
            assert float(got[at]) == value and int((got != 0).sum()) == 1


def test_infinities_stay_with_their_expert():
    """Rows of a neighbouring expert share a tile's loads; theirs may hold anything."""
    counts = [40, 30, 50, 0, 10]
    Z = sum(counts)
    for rows in (1, 20):  # on both sides of the choice of tiles
        c = [n * rows for n in counts]
        plan = _plan(c)
        xs, W = _randn((Z * rows, 96), torch.bfloat16, 1), _randn((5, 136, 96), torch.bfloat16, 2)
        gys = _randn((Z * rows, 136), torch.bfloat16, 3)
        a, b = c[0], c[0] + c[1]
        xs[a:b], gys[a:b], W[1] = math.nan, math.inf, -math.inf
        ys = plan.matmul(xs, W)
        gxs, gW = plan.matmul_backward(gys, xs, W)
        for t in (ys, gxs):
            assert bool(torch.isfinite(t[:a]).all()) and bool(torch.isfinite(t[b:]).all()) and not bool(torch.isfinite(t[a:b]).any())
        ok = torch.isfinite(gW).flatten(1).all(1)
        assert ok.tolist() == [True, False, True, True, True] and bool((gW[3] == 0).all())


def test_strides_and_alignment():
    counts = [33, 0, 90]
    plan, Z = _plan(counts), 123
    wide, stack, gwide = _randn((Z, 300), torch.bfloat16, 1), _randn((3, 90, 240), torch.bfloat16, 2), _randn((Z, 200), torch.bfloat16, 3)
    for skip in (0, 1, 8):
        _check(plan, counts, wide[:, skip:skip + 104], stack[:, skip:skip + 80, skip:skip + 104], gwide[:, skip:skip + 80])
    _check(plan, counts, _randn((104, Z), torch.float16, 1).t(), _randn((3, 104, 80), torch.float16, 2).transpose(1, 2),
           torch.ones((1, 1), dtype=torch.float16, device="cuda").expand(Z, 80))
    _check(plan, counts, wide[:, :104], stack[:1, :80, :104].expand(3, 80, 104), gwide[:, :80])


def test_gradients_against_differences():
    """The products are linear: differences of 64-bit sums over whole steps equal the gradients up to their rounding."""
    counts = [5, 12]
    plan = _plan(counts)
    xs, W, g = _randn((17, 24), torch.float16, 1), _randn((2, 16, 24), torch.float16, 2), _randn((17, 16), torch.float16, 3)
    gxs, gW = plan.matmul_backward(g, xs, W)
    e = torch.tensor([0] * 5 + [1] * 12, device="cuda")

    def f(x, w):
        return float((torch.einsum("snk,sk->sn", w[e], x) * g.double()).sum())

    x0, w0 = xs.double(), W.double()
    for s, k, n in ((0, 0, 0), (4, 23, 15), (5, 7, 8), (16, 1, 3)):
        dx = torch.zeros_like(x0)
        dx[s, k] = 0.5
        assert abs((f(x0 + dx, w0) - f(x0 - dx, w0)) - float(gxs[s, k])) <= 2.0 ** -10 * abs(float(gxs[s, k])) + 1e-4
        dw = torch.zeros_like(w0)
        dw[int(e[s]), n, k] = 0.5
        assert abs((f(x0, w0 + dw) - f(x0, w0 - dw)) - float(gW[e[s], n, k])) <= 2.0 ** -10 * abs(float(gW[e[s], n, k])) + 1e-4


def test_no_rows():
    from paper_2606_20855_gb300 import DeviceCSR, Routing
    R = DeviceCSR(4, 3, torch.zeros(5, dtype=torch.int64, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"),
                  torch.empty(0, device="cuda"))
    plan = Routing(R)
    x, W = torch.empty((0, 16), dtype=torch.bfloat16, device="cuda"), torch.ones((3, 24, 16), dtype=torch.bfloat16, device="cuda")
    assert plan.matmul(x, W).shape == (0, 24)
    gxs, gW = plan.matmul_backward(torch.empty((0, 24), dtype=torch.bfloat16, device="cuda"), x, W)
    assert gxs.shape == (0, 16) and bool((gW == 0).all())
    plan = _plan([2, 0, 3])
    for N, K in ((8, 0), (0, 8), (0, 0)):
        x, W = torch.ones((5, K), dtype=torch.bfloat16, device="cuda"), torch.ones((3, N, K), dtype=torch.bfloat16, device="cuda")
        assert torch.equal(plan.matmul(x, W), torch.zeros((5, N), dtype=torch.bfloat16, device="cuda"))
        gxs, gW = plan.matmul_backward(torch.ones((5, N), dtype=torch.bfloat16, device="cuda"), x, W)
        assert torch.equal(gxs, torch.zeros((5, K), dtype=torch.bfloat16, device="cuda")) and gW.shape == (3, N, K)


def test_equal_inputs_give_equal_bits():
    counts = [300, 2, 450]
    plan = _plan(counts)
    xs, W, g = _randn((752, 200), torch.bfloat16, 1), _randn((3, 320, 200), torch.bfloat16, 2), _randn((752, 320), torch.bfloat16, 3)
    first = (plan.matmul(xs, W), *plan.matmul_backward(g, xs, W))
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, (plan.matmul(xs, W), *plan.matmul_backward(g, xs, W))))


def test_refusals():
    from paper_2606_20855_gb300 import _abi
    plan = _plan([3, 4])
    x, W = torch.zeros((7, 16), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 8, 16), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        plan.matmul(x[:6], W)
    with pytest.raises(ValueError):
        plan.matmul(x, W[:1])
    with pytest.raises(ValueError):
        plan.matmul(x, W[:, :, :8])
    with pytest.raises(TypeError):
        plan.matmul(x, W.half())
    with pytest.raises(_abi.WsError) as e:
        plan.matmul(x.float(), W.float())
    assert e.value.status_name == "WS_ERR_DTYPE"
    with pytest.raises(ValueError):
        plan.matmul_backward(torch.zeros((7, 9), dtype=torch.bfloat16, device="cuda"), x, W)
    def call(ptr, room, size):
        _abi.ws_routing_matmul(plan._r, ptr, 16, W.data_ptr(), 16, 128, 8, 16, out.data_ptr(), 8, _abi.WS_BF16, room, size, 0)

    out, room = torch.zeros((7, 8), dtype=torch.bfloat16, device="cuda"), torch.zeros(1024, dtype=torch.uint8, device="cuda")
    for ptr, at, size in ((x.data_ptr() + 2, 0, 0), (x.data_ptr() + 2, room.data_ptr(), 16), (x.data_ptr() + 2, room.data_ptr() + 8, 512),
                          (x.data_ptr() + 1, room.data_ptr(), 1024)):  # no room for an aligned copy; odd address
        with pytest.raises(_abi.WsError) as e:
            call(ptr, at, size)
        assert e.value.status_name == "WS_ERR_INVALID_ARG"
