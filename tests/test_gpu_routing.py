"""Routing matrices on the GPU: choice of experts, the sort by expert, rows there and back, and their gradients,
against plain 64-bit computations.

Tolerances.  u is the unit roundoff of the result's type (2^-24, 2^-8, 2^-11).  A result rounded once from a 32-bit sum of n
terms is off by at most u |y| + n 2^-24 sum |terms|; weights are a quotient of exponentials (2 units each, CUDA's expf) and
a sum of n of them, so 8 + n units of 2^-24 bound them.
"""
from __future__ import annotations

import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -24}  # smallest step of halves near zero
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(shape, dt, seed):
    return torch.randn(shape, generator=_gen(seed), device="cuda").to(dt)


def _near(got, want, mass, n, dt):
    """|got - want| within one rounding to dt and n 32-bit roundings of terms that sum to `mass`."""
    want = want.double()
    bound = U[dt] * want.abs() + (n + 2) * 2.0 ** -24 * mass + TINY[dt]
    bad = (got.double() - want).abs() > bound
    assert not bool(bad.any()), (got[bad][:4], want[bad][:4])


# ------------------------------------------------------------------ choice


def _choice(x, k, normalize):
    """(columns, weights, 64-bit shares of all columns) by a stable sort."""
    x = x.double()
    cols = torch.sort(torch.where(x.isnan(), math.inf, x), dim=1, descending=True, stable=True).indices[:, :k].sort(1).values
    top = x.max(1, keepdim=True).values
    e = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    picked = e.gather(1, cols)
    total = (picked if normalize else e).sum(1, keepdim=True)
    total = torch.where(total == 0, 1.0, total)
    return cols, picked / total, e / total


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 64, 8), (3, 2, 2), (33, 60, 4), (1000, 257, 8), (7, 1000, 32),
                                   (50, 1024, 5), (2049, 33, 1), (9, 31, 31)])
@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("normalize", [True, False])
def test_choice_and_gradient(T, E, k, dt, normalize):
    from paper_2606_20855_gb300 import topk_route, topk_route_backward
    x = _randn((T, E), dt, T + E + k) * 2
    if E > 4:
        x[torch.rand((T, E), generator=_gen(5), device="cuda") < 0.1] = -math.inf
    x[T // 2] = -math.inf  # nothing left to choose from
    R = topk_route(x, k, normalize)
    cols, v, p = _choice(x, k, normalize)
    assert torch.equal(R.rowptr, torch.arange(T + 1, device="cuda") * k)
    assert torch.equal(R.colidx.view(T, k).long(), cols)
    got = R.vals.view(T, k).double()
    assert bool(((got - v).abs() <= (8 + E) * 2.0 ** -24 * v).all())
    assert bool((got[T // 2] == 0).all())
    g = _randn(T * k, torch.float32, 3)
    gx = topk_route_backward(x, R, g, normalize)
    g64 = g.view(T, k).double()
    a = (v * g64).sum(1, keepdim=True)
    scattered = torch.zeros_like(p).scatter(1, cols, g64)
    if normalize:
        want = torch.zeros_like(p).scatter(1, cols, v * (g64 - a))
        mass = torch.zeros_like(p).scatter(1, cols, v * (g64.abs() + (v * g64.abs()).sum(1, keepdim=True)))
    else:
        want = p * (scattered - a)
        mass = p * (scattered.abs() + (v * g64.abs()).sum(1, keepdim=True))
    assert gx.dtype == dt
    _near(gx, want, mass, 16 + E, dt)


def test_choice_of_ties_zeros_and_nan():
    from paper_2606_20855_gb300 import topk_route
    x = torch.zeros((4, 200), device="cuda")
    x[0, 100:] = -0.0  # equal to +0: the lowest columns win
    x[1, ::2] = 1.0
    x[2, 150] = math.nan
    x[3, 7] = math.inf
    R = topk_route(x, 4)
    c = R.colidx.view(4, 4).tolist()
    assert c == [[0, 1, 2, 3], [0, 2, 4, 6], [0, 1, 2, 150], [0, 1, 2, 7]]
    v = R.vals.view(4, 4)
    assert bool((v[:2] == 0.25).all()) and bool(v[2].isnan().all()) and bool(v[3].isnan().all())
    bf = torch.randint(0, 3, (300, 96), generator=_gen(0), device="cuda").to(torch.bfloat16)
    assert torch.equal(topk_route(bf, 6).colidx.view(300, 6).long(), _choice(bf, 6, True)[0])


def test_choice_of_strided_logits():
    from paper_2606_20855_gb300 import topk_route, topk_route_backward
    big = _randn((40, 131), torch.bfloat16, 1)
    for x in (big[:, 1:65], big[::2, 3:67], big.t()[:64].t(), big[:1].expand(40, 131)):
        a, b = topk_route(x, 5, False), topk_route(x.contiguous(), 5, False)
        assert torch.equal(a.colidx, b.colidx) and torch.equal(a.vals, b.vals)
        g = _randn(a.nnz, torch.float32, 2)
        assert torch.equal(topk_route_backward(x, a, g, False), topk_route_backward(x.contiguous(), b, g, False))


def test_gradient_of_choice_against_differences():
    """Central differences of sum g v in 64 bits around 32-bit logits, the chosen columns held fixed."""
    from paper_2606_20855_gb300 import topk_route, topk_route_backward
    x = _randn((5, 12), torch.float32, 8)
    g = _randn(5 * 3, torch.float32, 9)
    for normalize in (True, False):
        R = topk_route(x, 3, normalize)
        gx = topk_route_backward(x, R, g, normalize).double()
        cols = R.colidx.view(5, 3).long()

        def f(z):
            e = torch.exp(z)
            picked = e.gather(1, cols)
            return (picked / (picked if normalize else e).sum(1, keepdim=True) * g.view(5, 3).double()).sum(1)

        for j in range(12):
            d = torch.zeros_like(gx)
            d[:, j] = 1e-5
            slope = (f(x.double() + d) - f(x.double() - d)) / 2e-5
            assert float((slope - gx[:, j]).abs().max()) < 1e-6


# ------------------------------------------------------------------ sort


def _matrix(T, E, lens, seed, vals=None):
    """A routing matrix with lens[i] distinct columns in row i."""
    from paper_2606_20855_gb300 import DeviceCSR
    lens = torch.as_tensor(lens, device="cuda")
    order = torch.rand((T, E), generator=_gen(seed), device="cuda").argsort(1)
    keep = torch.zeros((T, E), dtype=torch.bool, device="cuda")
    keep.scatter_(1, order, torch.arange(E, device="cuda")[None, :] < lens[:, None])
    rowptr = torch.zeros(T + 1, dtype=torch.int64, device="cuda")
    rowptr[1:] = torch.cumsum(keep.sum(1), 0)
    colidx = keep.nonzero()[:, 1].to(torch.int32)
    return DeviceCSR(T, E, rowptr, colidx, _randn(colidx.numel(), torch.float32, seed + 1))


def _lens(T, E, kind, seed):
    if kind == "ragged":
        return torch.randint(0, min(E, 9) + 1, (T,), generator=_gen(seed), device="cuda")
    if kind == "sparse":  # most rows empty, some full
        full = torch.rand(T, generator=_gen(seed), device="cuda") < 0.05
        return torch.where(full, E, 0)
    return torch.full((T,), min(E, int(kind)), device="cuda")


SHAPES = [(1, 1, "1"), (1, 64, "8"), (31, 5, "ragged"), (32, 64, "4"), (513, 3, "2"), (1024, 60, "8"), (1025, 60, "8"),
          (1537, 1024, "2"), (5000, 257, "ragged"), (700, 1024, "sparse"), (90_001, 16, "ragged"), (200_003, 130, "sparse")]


@pytest.mark.parametrize("T,E,kind", SHAPES)
def test_sorted_by_column(T, E, kind):
    from paper_2606_20855_gb300 import Routing
    R = _matrix(T, E, _lens(T, E, kind, T), T + E)
    plan = Routing(R, validate=True)
    row = torch.repeat_interleave(torch.arange(T, device="cuda"), R.rowptr[1:] - R.rowptr[:-1])
    col, entries = torch.sort(R.colidx, stable=True)
    assert torch.equal(plan.offsets, torch.searchsorted(col, torch.arange(E + 1, dtype=torch.int32, device="cuda")))
    assert torch.equal(plan.rows.long(), row[entries])
    assert torch.equal(plan.entries.long(), entries)
    assert torch.equal(plan.slots[entries].long(), torch.arange(R.nnz, device="cuda"))


@pytest.mark.parametrize("T,E,kind", [(2929, 1024, "ragged"), (2930, 1024, "8"), (12_000, 300, "ragged"), (23_437, 128, "4"),
                                      (23_438, 128, "sparse"), (100_001, 33, "ragged")])
def test_many_rows_and_columns_sorted(T, E, kind):
    """Both sides of the size from which tiles have more warps."""
    test_sorted_by_column(T, E, kind)


@pytest.mark.parametrize("T,E", [(0, 4), (0, 0), (5, 0), (5, 7), (3000, 7)])
def test_no_entries(T, E):
    from paper_2606_20855_gb300 import Routing
    R = _matrix(T, E, [0] * T, 0) if T and E else _matrix(max(T, 1), max(E, 1), [0] * max(T, 1), 0)
    R.nrows, R.ncols, R.rowptr = T, E, torch.zeros(T + 1, dtype=torch.int64, device="cuda")
    plan = Routing(R)
    assert torch.equal(plan.offsets, torch.zeros(E + 1, dtype=torch.int64, device="cuda"))
    assert plan.dispatch(torch.ones((T, 8), device="cuda")).shape == (0, 8)
    y = plan.combine(torch.ones((0, 8), device="cuda"))
    assert torch.equal(y, torch.zeros((T, 8), device="cuda"))
    gys, gvals = plan.combine_backward(torch.ones((T, 8), device="cuda"), torch.ones((0, 8), device="cuda"))
    assert gys.shape == (0, 8) and gvals.shape == (0,)


def test_columns_out_of_range_take_no_part():
    from paper_2606_20855_gb300 import DeviceCSR, Routing
    for T in (4, 3000):
        rowptr = torch.arange(T + 1, device="cuda") * 2
        col = torch.tensor([0, 3], dtype=torch.int32, device="cuda").repeat(T)
        col[5] = 99
        col[2] = -1
        R = DeviceCSR(T, 4, rowptr, col, torch.ones(2 * T, device="cuda"))
        plan = Routing(R)
        assert plan.slots[5] == -1 and plan.slots[2] == -1
        assert int(plan.offsets[-1]) == 2 * T - 2 and plan.rows[-2:].tolist() == [-1, -1]
        x = _randn((T, 24), torch.float32, 0)
        xs = plan.dispatch(x)
        assert torch.equal(xs[:-2], x[plan.rows[:-2].long()]) and bool((xs[-2:] == 0).all())
        y = plan.combine(torch.full_like(xs, 3.0))
        assert torch.equal(y[:4, 0], torch.tensor([6.0, 3.0, 3.0, 6.0], device="cuda"))
        gys, gvals = plan.combine_backward(x, xs)
        assert bool((gys[-2:] == 0).all()) and gvals[5] == 0 and gvals[2] == 0
        # a row pointer that leaves the arrays is read inside them
        R.rowptr = rowptr.clone()
        R.rowptr[1], R.rowptr[T - 1] = -5, 10 ** 12
        Routing(R).dispatch(x)
    torch.cuda.synchronize()


# ------------------------------------------------------------------ rows there and back


@pytest.mark.parametrize("T,E,kind", [(1, 8, "2"), (33, 64, "8"), (700, 17, "ragged"), (1500, 40, "sparse"), (4097, 9, "5")])
@pytest.mark.parametrize("H", [1, 7, 48, 1001, 2048])
@pytest.mark.parametrize("dt", TYPES)
def test_rows_there_and_back(T, E, kind, H, dt):
    from paper_2606_20855_gb300 import Routing
    R = _matrix(T, E, _lens(T, E, kind, 3 * T), T)
    plan = Routing(R)
    rows, entries, Z = plan.rows.long(), plan.entries.long(), R.nnz
    x, ys = _randn((T, H), dt, 1), _randn((Z, H), dt, 2)
    gy, gxs = _randn((T, H), dt, 3), _randn((Z, H), dt, 4)
    assert torch.equal(plan.dispatch(x), x[rows])
    v = R.vals[entries].double()[:, None]
    zero = torch.zeros((T, H), dtype=torch.float64, device="cuda")
    most = int((R.rowptr[1:] - R.rowptr[:-1]).max())
    terms = v * ys.double()
    _near(plan.combine(ys), zero.index_add(0, rows, terms), zero.index_add(0, rows, terms.abs()), most, dt)
    _near(plan.dispatch_backward(gxs), zero.index_add(0, rows, gxs.double()), zero.index_add(0, rows, gxs.double().abs()), most, dt)
    gys, gvals = plan.combine_backward(gy, ys)
    _near(gys, v * gy.double()[rows], 0.0, 0, dt)
    prod = gy.double()[rows] * ys.double()
    want = torch.empty(Z, dtype=torch.float64, device="cuda")
    mass = torch.empty_like(want)
    want[entries], mass[entries] = prod.sum(1), prod.abs().sum(1)
    _near(gvals, want, mass, H, torch.float32)


def test_rows_with_strides_and_offsets():
    """Rows inside wider matrices, at every alignment; broadcast and transposed gradients."""
    from paper_2606_20855_gb300 import Routing
    R = _matrix(130, 12, _lens(130, 12, "3", 0), 7)
    plan = Routing(R)
    for dt in TYPES:
        for skip in (0, 1, 2, 4, 8):
            wide = _randn((130, 96), dt, skip)
            x = wide[:, skip:skip + 64]
            assert torch.equal(plan.dispatch(x), plan.dispatch(x.contiguous()))
            ys = _randn((R.nnz, 80), dt, 1)[:, skip:skip + 64]
            assert torch.equal(plan.combine(ys), plan.combine(ys.contiguous()))
            for a, b in zip(plan.combine_backward(x, ys), plan.combine_backward(x.contiguous(), ys.contiguous())):
                assert torch.equal(a, b)
        one = torch.ones((1, 1), dtype=dt, device="cuda").expand(130, 64)
        assert torch.equal(plan.combine_backward(one, ys)[0], plan.combine_backward(one.contiguous(), ys)[0])
        t = _randn((64, 130), dt, 2).t()
        assert torch.equal(plan.dispatch(t), t.contiguous()[plan.rows.long()])


def test_infinities_stay_in_their_rows():
    from paper_2606_20855_gb300 import Routing
    R = _matrix(50, 6, [2] * 50, 3)
    plan = Routing(R)
    ys = _randn((100, 32), torch.bfloat16, 0)
    ys[10] = math.inf
    ys[20] = math.nan
    y = plan.combine(ys)
    hit = torch.zeros(50, dtype=torch.bool, device="cuda")
    hit[plan.rows[[10, 20]].long()] = True
    assert torch.equal(~torch.isfinite(y).all(1), hit)


def test_equal_inputs_give_equal_bits_and_values_are_read_anew():
    from paper_2606_20855_gb300 import Routing
    R = _matrix(3000, 64, _lens(3000, 64, "8", 0), 1)
    ys = _randn((R.nnz, 256), torch.bfloat16, 0)
    a, b = Routing(R), Routing(R)
    assert torch.equal(a.combine(ys), b.combine(ys))
    assert torch.equal(a.slots, b.slots) and torch.equal(a.rows, b.rows)
    y = a.combine(ys)
    R.vals.mul_(2)  # exact
    assert torch.equal(a.combine(ys).float(), 2 * y.float())


def test_streams():
    """Work on another stream than the tensors' own, and a plan used on another stream than it was built on."""
    from paper_2606_20855_gb300 import Routing, topk_route
    logits = _randn((5000, 64), torch.float32, 0)
    x = _randn((5000, 512), torch.bfloat16, 1)
    R0 = topk_route(logits, 4)
    want = Routing(R0).dispatch(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    R = topk_route(logits, 4, stream=s)
    plan = Routing(R, stream=s)
    xs = plan.dispatch(x, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(R.vals, R0.vals) and torch.equal(xs, want)
    assert torch.equal(plan.dispatch(x), want)
    with torch.cuda.stream(s):
        s.wait_stream(torch.cuda.default_stream())
        again = plan.combine(want)
    s.synchronize()
    assert torch.equal(again, Routing(R0).combine(want))


def test_graph_capture():
    from paper_2606_20855_gb300 import Routing, topk_route
    logits, x = _randn((2000, 32), torch.float32, 0), _randn((2000, 128), torch.bfloat16, 1)

    def step():
        plan = Routing(topk_route(logits, 2))
        return plan.combine(plan.dispatch(x))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = step()
    logits.copy_(_randn((2000, 32), torch.float32, 5))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, step())
    _near(y, x.double(), 4 * x.double().abs(), 8, torch.bfloat16)  # weights that sum to one over equal rows


def test_refusals():
    from paper_2606_20855_gb300 import DeviceCSR, Routing, _abi, topk_route, topk_route_backward
    x = torch.zeros((4, 8), device="cuda")
    for k in (0, 9, -1):
        with pytest.raises(ValueError):
            topk_route(x, k)
    with pytest.raises(ValueError):
        topk_route(torch.zeros((4, 64), device="cuda"), 33)
    with pytest.raises(ValueError):
        topk_route(x[0], 2)
    with pytest.raises(TypeError):
        topk_route(x.double(), 2)
    with pytest.raises(TypeError):
        topk_route(x.cpu(), 2)
    with pytest.raises(_abi.WsError) as e:
        topk_route(torch.zeros((4, 1025), device="cuda"), 2)
    assert e.value.status_name == "WS_ERR_OVERFLOW"
    R = topk_route(x, 2)
    with pytest.raises(ValueError):
        topk_route_backward(x[:, :7], R, R.vals)
    with pytest.raises(TypeError):
        topk_route_backward(x, R, R.vals.double())
    plan = Routing(R)
    with pytest.raises(ValueError):
        plan.dispatch(torch.zeros((5, 8), device="cuda"))
    with pytest.raises(TypeError):
        plan.dispatch(torch.zeros((4, 8), dtype=torch.float64, device="cuda"))
    with pytest.raises(TypeError):
        plan.combine_backward(torch.zeros((4, 8), device="cuda"), torch.zeros((8, 8), dtype=torch.float16, device="cuda"))
    with pytest.raises(ValueError):
        plan.combine_backward(torch.zeros((4, 9), device="cuda"), torch.zeros((8, 8), device="cuda"))
    with pytest.raises(TypeError):
        Routing(DeviceCSR(4, 8, R.rowptr, R.colidx, R.vals.double()))
    with pytest.raises(ValueError):
        Routing(DeviceCSR(5, 8, R.rowptr, R.colidx, R.vals))
    with pytest.raises(_abi.WsError) as e:
        Routing(DeviceCSR(4, 1025, R.rowptr, R.colidx, R.vals))
    assert e.value.status_name == "WS_ERR_OVERFLOW"
    bad = R.colidx.clone()
    bad[:2] = 7
    with pytest.raises(_abi.WsError) as e:
        Routing(DeviceCSR(4, 8, R.rowptr, bad, R.vals), validate=True)
    assert e.value.status_name == "WS_ERR_INVALID_CSR"
