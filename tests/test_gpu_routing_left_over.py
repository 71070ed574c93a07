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
