"""Refusals of the calls on routing matrices at the C entry: argument errors are found on the host, before any CUDA call."""
from __future__ import annotations

import ctypes

import pytest

from paper_2606_20855_gb300 import _abi
from paper_2606_20855_gb300 import build as pkg_build

P = 1 << 20  # an address that is never used


@pytest.fixture(scope="module", autouse=True)
def lib():
    pkg_build.build()
    return _abi.load()


def _refused(status, f, *args):
    with pytest.raises(_abi.WsError) as e:
        f(*args)
    assert e.value.status_name == status and str(e.value)


def _routing(nrows=4, ncols=3, nnz=8, **kv):
    fields = dict(nrows=nrows, ncols=ncols, nnz=nnz, rowptr=P, colidx=P, vals=P, offsets=P, rows=P, entries=P, slots=P, status=P)
    fields.update(kv)
    return ctypes.byref(_abi.WsRouting(*(fields[n] for n, _ in _abi.WsRouting._fields_)))


def test_choice():
    def call(rows=4, cols=8, ld=8, dtype=_abi.WS_F32, k=2, logits=P, rowptr=P, colidx=P, vals=P):
        _abi.ws_topk_route(logits, rows, cols, ld, dtype, k, True, rowptr, colidx, vals, 0)

    for kv in (dict(rows=-1), dict(cols=0), dict(k=0), dict(k=9), dict(cols=64, ld=64, k=33), dict(ld=7), dict(logits=0),
               dict(rowptr=0), dict(colidx=0), dict(vals=0), dict(logits=P + 1)):
        _refused("WS_ERR_INVALID_ARG", lambda kv=kv: call(**kv))
    _refused("WS_ERR_DTYPE", lambda: call(dtype=_abi.WS_F64))
    _refused("WS_ERR_OVERFLOW", lambda: call(cols=1025, ld=1025))
    _refused("WS_ERR_OVERFLOW", lambda: call(rows=2 ** 31))

    def back(rows=4, cols=8, ld=8, dtype=_abi.WS_BF16, k=2, normalize=True, logits=P, colidx=P, vals=P, gvals=P, out=P, ldg=8):
        _abi.ws_topk_route_backward(logits, rows, cols, ld, dtype, k, normalize, colidx, vals, gvals, out, ldg, 0)

    for kv in (dict(k=0), dict(colidx=0), dict(gvals=0), dict(out=0), dict(ldg=7), dict(out=P + 1), dict(normalize=False, logits=0),
               dict(normalize=False, ld=7)):
        _refused("WS_ERR_INVALID_ARG", lambda kv=kv: back(**kv))
    _refused("WS_ERR_DTYPE", lambda: back(dtype=7))


def test_plan():
    for r, status in ((None, "WS_ERR_INVALID_ARG"), (_routing(nrows=-1), "WS_ERR_INVALID_ARG"), (_routing(offsets=0), "WS_ERR_INVALID_ARG"),
                      (_routing(slots=0), "WS_ERR_INVALID_ARG"), (_routing(status=0), "WS_ERR_INVALID_ARG"), (_routing(ncols=1025), "WS_ERR_OVERFLOW"),
                      (_routing(nnz=2 ** 31), "WS_ERR_OVERFLOW"), (_routing(nrows=0), "WS_ERR_SHAPE"), (_routing(ncols=0), "WS_ERR_SHAPE")):
        _refused(status, _abi.ws_routing_build, r, 0, 0, 0)


def test_rows():
    r = _routing()
    for f in (_abi.ws_routing_dispatch, _abi.ws_routing_dispatch_backward, _abi.ws_routing_combine):
        _refused("WS_ERR_INVALID_ARG", f, None, P, 16, P, 16, 16, _abi.WS_F32, 0)
        _refused("WS_ERR_INVALID_ARG", f, r, 0, 16, P, 16, 16, _abi.WS_F32, 0)
        _refused("WS_ERR_INVALID_ARG", f, r, P, 15, P, 16, 16, _abi.WS_F32, 0)
        _refused("WS_ERR_INVALID_ARG", f, r, P, 16, P + 2, 16, 16, _abi.WS_F32, 0)
        _refused("WS_ERR_INVALID_ARG", f, r, P, 16, P, 16, -1, _abi.WS_F32, 0)
        _refused("WS_ERR_DTYPE", f, r, P, 16, P, 16, 16, _abi.WS_F64, 0)
        _refused("WS_ERR_OVERFLOW", f, r, P, 2 ** 25, P, 2 ** 25, 2 ** 25, _abi.WS_F32, 0)
    _refused("WS_ERR_INVALID_ARG", _abi.ws_routing_combine, _routing(vals=0), P, 16, P, 16, 16, _abi.WS_F32, 0)
    _refused("WS_ERR_INVALID_ARG", _abi.ws_routing_combine_backward, r, P, 16, P, 16, P, 16, 0, 16, _abi.WS_F32, 0)


def test_products():
    def call(r=None, xs=P, ldx=16, W=P, ldw=16, stride=128, N=8, K=16, ys=P, ldy=8, dtype=_abi.WS_BF16, room=0, size=0):
        _abi.ws_routing_matmul(r or _routing(), xs, ldx, W, ldw, stride, N, K, ys, ldy, dtype, room, size, 0)

    for kv in (dict(xs=0), dict(W=0), dict(ys=0), dict(N=-1), dict(ldy=7), dict(xs=P + 1), dict(ldx=-8), dict(stride=-128)):
        _refused("WS_ERR_INVALID_ARG", lambda kv=kv: call(**kv))
    for dtype in (_abi.WS_F32, _abi.WS_F64, 9):
        _refused("WS_ERR_DTYPE", lambda d=dtype: call(dtype=d))
    _refused("WS_ERR_OVERFLOW", lambda: call(K=2 ** 25, ldx=2 ** 25, ldw=2 ** 25))
    with pytest.raises(_abi.WsError):
        _abi.ws_routing_matmul_backward(_routing(), 0, 8, P, 16, P, 16, 128, 8, 16, P, 16, P, 16, 128, _abi.WS_BF16, 0, 0, 0)


def test_adapters():
    def call(T=4, L=3, nnz=4, K=16, r=8, N=24, dtype=_abi.WS_F16, room=P, size=1 << 16, **kv):
        f = dict(rowptr=P, colidx=P, vals=P, x=P, ldx=K, A=P, lda=K, sA=r * K, B=P, ldb=r, sB=N * r, base=P, ldbase=N, y=P, ldy=N)
        f.update(kv)
        packed = _abi.ADAPTERS_CALL.pack(T, L, nnz, f["rowptr"], f["colidx"], f["vals"], K, r, N, f["x"], f["ldx"], f["A"], f["lda"],
                                         f["sA"], f["B"], f["ldb"], f["sB"], f["base"], f["ldbase"], f["y"], f["ldy"], dtype)
        _abi.ws_adapters(packed, room, size, 0)

    for kv in (dict(T=-1), dict(rowptr=0), dict(colidx=0), dict(x=0), dict(A=0), dict(B=0), dict(y=0), dict(ldy=23), dict(base=P + 1),
               dict(room=0), dict(size=16), dict(room=P + 8), dict(ldx=-1)):
        _refused("WS_ERR_INVALID_ARG", lambda kv=kv: call(**kv))
    _refused("WS_ERR_DTYPE", lambda: call(dtype=_abi.WS_F32))
    _refused("WS_ERR_OVERFLOW", lambda: call(r=5000))
    _refused("WS_ERR_SHAPE", lambda: call(L=0))
    assert _abi.ws_adapters_scratch(0, 8) == 16 and _abi.ws_adapters_scratch(10, 9) == 16 + 10 * 16 * 16
    _abi.ws_csr_destroy(0)


def test_16_bit_values_are_not_csr_values(lib):
    h = ctypes.c_void_p()
    for dtype in (_abi.WS_BF16, _abi.WS_F16):
        assert lib.ws_csr_create(ctypes.byref(h), 1, 1, 0, 8, None, None, dtype, 0, None) == 1
