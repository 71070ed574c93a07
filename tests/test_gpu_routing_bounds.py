"""Plans of routing matrices whose row pointer decreases or leaves the arrays: nothing outside the caller's arrays is written.

Which entries such a plan counts is modelled on the CPU: a warp goes through the entries from its first row's begin to its last row's
end and gives each to the row that a binary search over the rows' ends finds, so ranges that overlap count entries again.
"""
from __future__ import annotations

import ctypes

import numpy as np
import pytest
import torch

PAD = 1 << 14  # guard values on both sides of every array
MARK = 0x5A5A5A5A


def _marked(rowptr, colidx, ncols):
    """(row, column) of everything that the plan's warps mark."""
    nnz, T = colidx.size, rowptr.size - 1
    seen = set()
    for first in range(0, T, 32):
        rows = np.minimum(first + np.arange(32), T - 1)
        begin = np.clip(rowptr[rows], 0, nnz)
        end = np.maximum(begin, np.minimum(rowptr[rows + 1], nnz))
        begin = np.where(first + np.arange(32) < T, begin, end)
        x = np.arange(begin[0], max(begin[0], end[31]))
        n = np.zeros(x.size, dtype=np.int64)
        for step in (16, 8, 4, 2, 1):
            n += np.where(end[n + step - 1] <= x, step, 0)
        ok = (first + n < T) & (colidx[x] >= 0) & (colidx[x] < ncols)
        seen.update(zip((first + n[ok]).tolist(), colidx[x][ok].tolist()))
    return seen


def _offsets(seen, nnz, ncols):
    count = np.bincount(np.array([c for _, c in seen], dtype=np.int64), minlength=ncols)
    return np.minimum(np.concatenate([[0], np.cumsum(count)]), nnz)


def _case(name):
    """(row pointer, columns, number of columns)"""
    T, E, k = {"one low": (128, 64, 8), "restarts": (1024, 60, 2), "restarts, many columns": (1024, 1024, 4),
               "two launches": (5000, 33, 3), "two launches, many columns": (6000, 700, 2), "noise": (2000, 100, 4),
               "wide rows": (640, 16, 16), "one low, few columns": (2048, 8, 3)}[name]
    rng = np.random.default_rng(T + E)
    rowptr = np.arange(T + 1, dtype=np.int64) * k
    nnz = T * k
    if name.startswith("one low"):
        rowptr[32] = 0
    elif name == "noise":
        at = 32 * rng.integers(T // 64, T // 32, 40)
        rowptr[at] = rng.integers(-5, nnz, 40)
    else:
        nnz = 32 * k
        rowptr = (np.arange(T + 1, dtype=np.int64) % 32) * k
        rowptr[31::32] = nnz
        rowptr[-1] = nnz
    rows = np.argsort(rng.random((nnz // k, E)), axis=1)[:, :k]
    return rowptr, np.sort(rows, axis=1).reshape(-1).astype(np.int32), E


NAMES = ["one low", "restarts", "restarts, many columns", "two launches", "two launches, many columns", "noise", "wide rows",
         "one low, few columns"]


@pytest.mark.parametrize("name", NAMES)
def test_more_is_marked_than_there_are_entries(name):
    """The model itself: without a bound at nnz the plan's writes would leave its arrays."""
    rowptr, col, E = _case(name)
    assert len(_marked(rowptr, col, E)) > col.size


def test_model_of_a_proper_row_pointer():
    rowptr = np.array([0, 2, 2, 5, 6], dtype=np.int64)
    col = np.array([0, 2, 0, 1, 2, 1], dtype=np.int32)
    assert _marked(rowptr, col, 3) == {(0, 0), (0, 2), (2, 0), (2, 1), (2, 2), (3, 1)}


class _Guarded:
    """An int32 array on the GPU between guards."""

    def __init__(self, count):
        self.all = torch.full((count + 2 * PAD,), MARK, dtype=torch.int32, device="cuda")
        self.own = self.all[PAD:PAD + count]
        self.count = count

    def ptr(self):
        return self.own.data_ptr()

    def untouched(self):
        return bool((self.all[:PAD] == MARK).all()) and bool((self.all[PAD + self.count:] == MARK).all())


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_plan_stays_in_its_arrays(name):
    from paper_2606_20855_gb300 import _abi
    rowptr, col, E = _case(name)
    T, nnz = rowptr.size - 1, col.size
    want = _offsets(_marked(rowptr, col, E), nnz, E)
    rp, ci, v = torch.from_numpy(rowptr).cuda(), torch.from_numpy(col).cuda(), torch.ones(nnz, device="cuda")
    offsets, rows, entries, slots, status = (_Guarded(n) for n in (2 * (E + 1), nnz, nnz, nnz, 1))
    need = _abi.ws_routing_scratch(T, E)
    scratch = torch.zeros(max(need, 16), dtype=torch.uint8, device="cuda")
    r = _abi.WsRouting(T, E, nnz, rp.data_ptr(), ci.data_ptr(), v.data_ptr(), offsets.ptr(), rows.ptr(), entries.ptr(), slots.ptr(),
                       status.ptr())
    stream = torch.cuda.current_stream().cuda_stream
    _abi.ws_routing_build(ctypes.byref(r), scratch.data_ptr(), need, stream)
    torch.cuda.synchronize()
    for a in (offsets, rows, entries, slots, status):
        assert a.untouched()
    off = offsets.own.view(torch.int64).cpu().numpy()
    assert np.array_equal(off, want)
    assert bool(((rows.own >= -1) & (rows.own < T)).all()) and bool(((entries.own >= -1) & (entries.own < nnz)).all())
    assert bool(((slots.own >= -1) & (slots.own < nnz)).all())

    # rows there and back, and the products by column, stay in theirs
    for K, N in ((64, 48), (40, 136)):
        def dense(n, width):
            t = torch.full((n + 600, width), 77.0, dtype=torch.bfloat16, device="cuda")
            return t, t[:n]
        x, W = torch.ones((T, K), dtype=torch.bfloat16, device="cuda"), torch.ones((E, N, K), dtype=torch.bfloat16, device="cuda")
        (xs_all, xs), (ys_all, ys), (gx_all, gx) = dense(nnz, K), dense(nnz, N), dense(nnz, K)
        gW = torch.empty((E, N, K), dtype=torch.bfloat16, device="cuda")
        p = ctypes.byref(r)
        _abi.ws_routing_dispatch(p, x.data_ptr(), K, xs.data_ptr(), K, K, _abi.WS_BF16, stream)
        _abi.ws_routing_matmul(p, xs.data_ptr(), K, W.data_ptr(), K, N * K, N, K, ys.data_ptr(), N, _abi.WS_BF16, 0, 0, stream)
        _abi.ws_routing_matmul_backward(p, ys.data_ptr(), N, xs.data_ptr(), K, W.data_ptr(), K, N * K, N, K, gx.data_ptr(), K,
                                        gW.data_ptr(), K, N * K, _abi.WS_BF16, 0, 0, stream)
        torch.cuda.synchronize()
        for t in (xs_all, ys_all, gx_all):
            assert bool((t[nnz:] == 77.0).all())
        assert status.own.item() == 0
