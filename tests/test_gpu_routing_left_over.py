"""Entries of a routing matrix that take no part (columns out of range, entries of no row): every result is written there too."""
from __future__ import annotations

import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def _plan(counts, left_over):
    """A plan whose column e has counts[e] entries, one a row, and `left_over` entries without a column."""
    from paper_2606_20855_gb300 import DeviceCSR, Routing
    E, Z = len(counts), sum(counts) + left_over
    col = torch.cat([torch.repeat_interleave(torch.arange(E), torch.tensor(counts)), torch.full((left_over,), E)])
    col[col == E] = torch.where(torch.arange(left_over) % 2 == 0, -1, E + 5)
    col = col[torch.randperm(Z, generator=torch.Generator().manual_seed(Z))].to(torch.int32).cuda()
    return Routing(DeviceCSR(Z, E, torch.arange(Z + 1, device="cuda"), col, torch.ones(Z, device="cuda")))


# means of 2 to 700 entries a column, so that every kernel of the products is met
@pytest.mark.parametrize("counts,left_over", [([1], 1), ([2, 0, 3], 9), ([8], 700), ([9, 20, 0, 31], 5), ([0, 0], 40), ([60, 70], 60),
                                              ([300, 0, 250], 150), ([900, 1100], 300)])
@pytest.mark.parametrize("N,K", [(48, 64), (33, 24), (520, 264), (2304, 4608)])
def test_products_write_rows_behind_the_placed_entries(counts, left_over, N, K):
    from paper_2606_20855_gb300 import _abi
    plan = _plan(counts, left_over)
    placed, Z, E, bf = sum(counts), sum(counts) + left_over, len(counts), torch.bfloat16
    x, W, g = torch.ones((Z, (K + 7) // 8 * 8), dtype=bf, device="cuda"), torch.ones((E, N, (K + 7) // 8 * 8), dtype=bf, device="cuda"), \
        torch.ones((Z, (N + 7) // 8 * 8), dtype=bf, device="cuda")
    for pad in (0, 3):  # rows of the results at multiples of 16 bytes or not
        ys = torch.full((Z + 2, N + pad), math.nan, dtype=bf, device="cuda")
        gxs = torch.full((Z + 2, K + pad), math.nan, dtype=bf, device="cuda")
        stream = torch.cuda.current_stream().cuda_stream
        _abi.ws_routing_matmul(plan._r, x.data_ptr(), x.shape[1], W.data_ptr(), W.shape[2], W[0].numel(), N, K, ys.data_ptr(), N + pad,
                               _abi.WS_BF16, 0, 0, stream)
        _abi.ws_routing_matmul_backward(plan._r, g.data_ptr(), g.shape[1], 0, 0, W.data_ptr(), W.shape[2], W[0].numel(), N, K,
                                        gxs.data_ptr(), K + pad, 0, 0, 0, _abi.WS_BF16, 0, 0, stream)
        plan.wait()
        for t, width, value in ((ys, N, float(K)), (gxs, K, float(N))):
            value = float(torch.tensor(value).bfloat16())
            assert bool((t[:placed, :width] == value).all()) and bool((t[placed:Z, :width] == 0).all())
            assert bool(t[Z:].isnan().all()) and bool(t[:, width:].isnan().all())


@pytest.mark.parametrize("T,E,k", [(5, 7, 3), (700, 40, 4), (5000, 64, 2)])
@pytest.mark.parametrize("before,behind", [(0, 1), (0, 900), (300, 0), (17, 41)])
def test_entries_of_no_row(T, E, k, before, behind):
    """Arrays longer than the row pointer says, as a program has them that drops entries without reading their number back."""
    import ctypes
    from paper_2606_20855_gb300 import DeviceCSR, Routing, _abi
    g = torch.Generator().manual_seed(T)
    col = torch.rand((T, E), generator=g).argsort(1)[:, :k].sort(1).values.flatten().to(torch.int32)
    nnz, Z, H = T * k, before + T * k + behind, 40
    wide = torch.cat([torch.zeros(before, dtype=torch.int32), col, torch.full((behind,), E - 1, dtype=torch.int32)]).cuda()
    v = torch.rand(Z, generator=g).cuda()
    rowptr = torch.arange(T + 1, device="cuda") * k
    want = Routing(DeviceCSR(T, E, rowptr, col.cuda(), v[before:before + nnz].contiguous()))

    def filled(n, value, dt):
        return torch.full((n,), value, dtype=dt, device="cuda")

    rowptr = rowptr + before
    offsets, status = filled(E + 1, 7, torch.int64), filled(1, 7, torch.int32)
    rows, entries, slots = (filled(Z, 7, torch.int32) for _ in range(3))
    r = _abi.WsRouting(T, E, Z, rowptr.data_ptr(), wide.data_ptr(), v.data_ptr(), offsets.data_ptr(), rows.data_ptr(), entries.data_ptr(),
                       slots.data_ptr(), status.data_ptr())
    need, stream = _abi.ws_routing_scratch(T, E), torch.cuda.current_stream().cuda_stream
    room = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    p = ctypes.byref(r)
    _abi.ws_routing_build(p, room.data_ptr(), need, stream)
    assert torch.equal(offsets, want.offsets) and torch.equal(rows[:nnz], want.rows) and torch.equal(entries[:nnz], want.entries + before)
    assert bool((rows[nnz:] == -1).all()) and bool((entries[nnz:] == -1).all())
    assert torch.equal(slots[before:before + nnz], want.slots)
    assert bool((slots[:before] == -1).all()) and bool((slots[before + nnz:] == -1).all())

    gy, ys = (torch.randn((n, H), generator=g).cuda() for n in (T, Z))
    gys, gvals = torch.full((Z, H), math.nan, device="cuda"), filled(Z, math.nan, torch.float32)
    _abi.ws_routing_combine_backward(p, gy.data_ptr(), H, ys.data_ptr(), H, gys.data_ptr(), H, gvals.data_ptr(), H, _abi.WS_F32, stream)
    a, b = want.combine_backward(gy, ys[:nnz])
    assert torch.equal(gys[:nnz], a) and torch.equal(gvals[before:before + nnz], b)
    assert bool((gys[nnz:] == 0).all()) and bool((gvals[:before] == 0).all()) and bool((gvals[before + nnz:] == 0).all())
