"""Operations on sparse routing matrices: rows of dense matrices sent along a CSR matrix.

A routing matrix R (:class:`DeviceCSR`, float32 values, at most 1024 columns) has a row per token and a column per
expert.  A layer of experts is

    R = topk_route(logits, k)          # k experts of every token and their weights
    plan = Routing(R)                  # R transposed: the tokens sorted by expert
    xs = plan.dispatch(x)              # their rows in that order
    y = plan.combine(f(xs))            # the experts' rows summed back with R's values

where the experts' matrices may be ``plan.matmul(xs, W)``; the gradients are ``combine_backward``,
``dispatch_backward``, ``matmul_backward`` and ``topk_route_backward``.  All calls queue work on
the current stream, or on ``stream``, and return without waiting; none reads anything back.
"""
from __future__ import annotations

import contextlib
import ctypes

import torch

from . import _abi
from .spgemm import DeviceCSR

_ROW_DTYPES = {torch.float32: _abi.WS_F32, torch.bfloat16: _abi.WS_BF16, torch.float16: _abi.WS_F16}
_HERE = contextlib.nullcontext()


def _on(stream, *tensors):
    """Context in which results are allocated and work is queued on ``stream`` (None: the current one).  Inputs that
    came from another stream stay allocated until it is done with them."""
    if stream is None:
        return _HERE
    for t in tensors:
        t.record_stream(stream)
    return torch.cuda.stream(stream)


def _raw_stream(device) -> int:
    return torch._C._cuda_getCurrentRawStream(device.index)


def _dtype(t: torch.Tensor, name: str) -> int:
    dt = _ROW_DTYPES.get(t.dtype)
    if dt is None:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    return dt


def _matrix(t: torch.Tensor, name: str, rows: int | None, like: torch.Tensor | None = None) -> torch.Tensor:
    """A 2-D CUDA tensor whose rows have unit stride (copied if they have not)."""
    if not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dim() != 2 or (rows is not None and t.shape[0] != rows):
        raise ValueError(f"{name} must be 2-D" + (f" with {rows} rows" if rows is not None else "") +
                         f", got {tuple(t.shape)}")
    if like is not None and (t.dtype != like.dtype or t.device != like.device):
        raise TypeError(f"{name} must have the other matrix's type and device")
    n = t.shape[1]
    if (n > 1 and t.stride(1) != 1) or (t.shape[0] > 1 and t.stride(0) < n):
        return t.contiguous()
    return t


def _operand(t: torch.Tensor) -> torch.Tensor:
    """A matrix (or a stack of matrices) of 16-bit values whose rows start at multiples of 16 bytes: t itself, or a
    copy with longer rows where t's do not."""
    n = t.shape[-1]
    if t.data_ptr() % 16 == 0 and (n <= 1 or t.stride(-1) == 1) and \
            all(t.shape[i] == 1 or (t.stride(i) % 8 == 0 and t.stride(i) >= n) for i in range(t.dim() - 1)):
        return t
    out = torch.empty((*t.shape[:-1], (n + 7) // 8 * 8), dtype=t.dtype, device=t.device)[..., :n]
    return out.copy_(t)


def _ld8(t: torch.Tensor) -> int:
    return t.stride(-2) if t.shape[-2] > 1 else (t.shape[-1] + 7) // 8 * 8


def _ld(t: torch.Tensor) -> int:
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def topk_route(logits: torch.Tensor, k: int, normalize: bool = True, stream=None) -> DeviceCSR:
    """The routing matrix of a T x E tensor of logits: row i holds the k largest logits of row i (ties to the lowest
    column), by ascending column, with softmax weights over the chosen (``normalize``) or over all columns.  A logit
    of -inf has weight 0 and is chosen last; a row of nothing else has weights 0."""
    dt = _dtype(logits, "logits")
    with _on(stream, logits):
        x = _matrix(logits, "logits", None)
        (T, E), k, dev = x.shape, int(k), x.device
        if not 1 <= k <= min(E, 32):
            raise ValueError(f"k must be in 1..min(columns, 32), got {k} of {E}")
        rowptr = torch.empty(T + 1, dtype=torch.int64, device=dev)
        colidx = torch.empty(T * k, dtype=torch.int32, device=dev)
        vals = torch.empty(T * k, dtype=torch.float32, device=dev)
        _abi.ws_topk_route(x.data_ptr(), T, E, _ld(x), dt, k, normalize, rowptr.data_ptr(), colidx.data_ptr(),
                           vals.data_ptr(), _raw_stream(dev))
    return DeviceCSR(T, E, rowptr, colidx, vals)


def topk_route_backward(logits: torch.Tensor, R: DeviceCSR, grad_vals: torch.Tensor, normalize: bool = True,
                        stream=None) -> torch.Tensor:
    """Gradient of the logits from that of R's values, for ``R = topk_route(logits, k, normalize)``."""
    dt = _dtype(logits, "logits")
    with _on(stream, logits, R.colidx, R.vals, grad_vals):
        x = _matrix(logits, "logits", R.nrows)
        T, E = x.shape
        k = R.nnz // T if T else 1
        if E != R.ncols or k * T != R.nnz:
            raise ValueError("R is not the routing matrix of these logits")
        if grad_vals.dtype != torch.float32 or grad_vals.numel() != R.nnz or R.vals.dtype != torch.float32:
            raise TypeError("grad_vals must be float32, one for every value of R")
        g, vals = grad_vals.contiguous(), R.vals.contiguous()
        out = torch.empty((T, E), dtype=x.dtype, device=x.device)
        _abi.ws_topk_route_backward(x.data_ptr(), T, E, _ld(x), dt, k, normalize, R.colidx.data_ptr(),
                                    vals.data_ptr(), g.data_ptr(), out.data_ptr(), E, _raw_stream(x.device))
    return out


class Routing:
    """A routing matrix with its transpose: the entries of R sorted by column, rows in order within a column.

    ``offsets`` (int64 [E + 1]) is the first slot of every column, ``rows`` and ``entries`` (int32 [nnz]) are the row
    and the entry of R in every slot, ``slots`` (int32 [nnz]) is the slot of every entry.  Entries whose column is out
    of range have slot -1 and take no part; the slots they leave over come last, hold -1 and stand for zero rows.
    The object uses R's arrays as they are at every call: ``combine`` reads R's values then.
    """

    def __init__(self, R: DeviceCSR, validate: bool = False, stream=None):
        if R.vals.dtype != torch.float32:
            raise TypeError(f"a routing matrix has float32 values, got {R.vals.dtype}")
        for t, dt in ((R.rowptr, torch.int64), (R.colidx, torch.int32), (R.vals, torch.float32)):
            if t.dtype != dt or not t.is_cuda or not t.is_contiguous():
                raise TypeError("rowptr/colidx/vals must be contiguous CUDA int64/int32/float32 tensors")
        nnz, E = R.colidx.numel(), R.ncols
        if R.rowptr.numel() != R.nrows + 1 or R.vals.numel() != nnz:
            raise ValueError("rowptr must have nrows + 1 entries, and every column index a value")
        self.R, self.nnz, self.device = R, nnz, R.rowptr.device
        with _on(stream, R.rowptr, R.colidx, R.vals):
            raw = _raw_stream(self.device)
            if validate:
                _abi.ws_csr_destroy(R._handle(True, raw))
            scratch = _abi.ws_routing_scratch(R.nrows, E)
            # offsets, then rows, entries and slots, the status word, the scratch
            words = 2 * (E + 1) + 3 * nnz + 1
            self._buf = torch.empty(words + scratch // 4, dtype=torch.int32, device=self.device)
            at = self._buf.data_ptr()
            rows = at + 8 * (E + 1)
            self._c = _abi.WsRouting(R.nrows, E, nnz, R.rowptr.data_ptr(), R.colidx.data_ptr() or None,
                                     R.vals.data_ptr() or None, at, rows, rows + 4 * nnz, rows + 8 * nnz,
                                     rows + 12 * nnz)
            self._r = ctypes.byref(self._c)
            self._stream = raw
            _abi.ws_routing_build(self._r, at + 4 * words, scratch, raw)

    def _ints(self, i: int) -> torch.Tensor:
        at = 2 * (self.R.ncols + 1) + i * self.nnz
        return self._buf[at:at + self.nnz]

    @property
    def offsets(self) -> torch.Tensor:
        return self._buf[:2 * (self.R.ncols + 1)].view(torch.int64)

    @property
    def rows(self) -> torch.Tensor:
        return self._ints(0)

    @property
    def entries(self) -> torch.Tensor:
        return self._ints(1)

    @property
    def slots(self) -> torch.Tensor:
        return self._ints(2)

    def _queue(self) -> int:
        """The current stream; the plan's arrays stay allocated until it is done with them."""
        raw = _raw_stream(self.device)
        if raw != self._stream:
            s = torch.cuda.current_stream(self.device)
            for t in (self._buf, self.R.rowptr, self.R.colidx, self.R.vals):
                t.record_stream(s)
        return raw

    def dispatch(self, x: torch.Tensor, stream=None) -> torch.Tensor:
        """xs[slot] = x[row]: the rows of x (T x H) in slot order (nnz x H)."""
        dt = _dtype(x, "x")
        with _on(stream, x):
            x = _matrix(x, "x", self.R.nrows)
            H = x.shape[1]
            out = torch.empty((self.nnz, H), dtype=x.dtype, device=x.device)
            _abi.ws_routing_dispatch(self._r, x.data_ptr(), _ld(x), out.data_ptr(), H, H, dt, self._queue())
        return out

    def dispatch_backward(self, grad_xs: torch.Tensor, stream=None) -> torch.Tensor:
        """Gradient of x: gx[i] = sum of grad_xs over the slots of row i."""
        dt = _dtype(grad_xs, "grad_xs")
        with _on(stream, grad_xs):
            g = _matrix(grad_xs, "grad_xs", self.nnz)
            H = g.shape[1]
            out = torch.empty((self.R.nrows, H), dtype=g.dtype, device=g.device)
            _abi.ws_routing_dispatch_backward(self._r, g.data_ptr(), _ld(g), out.data_ptr(), H, H, dt, self._queue())
        return out

    def combine(self, ys: torch.Tensor, stream=None) -> torch.Tensor:
        """y[i] = sum over row i of R's value times ys[slot]."""
        dt = _dtype(ys, "ys")
        with _on(stream, ys):
            ys = _matrix(ys, "ys", self.nnz)
            H = ys.shape[1]
            out = torch.empty((self.R.nrows, H), dtype=ys.dtype, device=ys.device)
            _abi.ws_routing_combine(self._r, ys.data_ptr(), _ld(ys), out.data_ptr(), H, H, dt, self._queue())
        return out

    def combine_backward(self, grad_y: torch.Tensor, ys: torch.Tensor, stream=None):
        """Gradients of ys (value times grad_y's row) and of R's values (the products of grad_y's and ys's rows)."""
        dt = _dtype(ys, "ys")
        with _on(stream, ys, grad_y):
            ys = _matrix(ys, "ys", self.nnz)
            g = _matrix(grad_y, "grad_y", self.R.nrows, ys)
            H = ys.shape[1]
            if g.shape[1] != H:
                raise ValueError("grad_y and ys differ in the length of their rows")
            out = torch.empty((self.nnz, H), dtype=ys.dtype, device=ys.device)
            gvals = torch.empty(self.nnz, dtype=torch.float32, device=ys.device)
            _abi.ws_routing_combine_backward(self._r, g.data_ptr(), _ld(g), ys.data_ptr(), _ld(ys), out.data_ptr(), H,
                                             gvals.data_ptr(), H, dt, self._queue())
        return out, gvals

    def _experts(self, W: torch.Tensor, like: torch.Tensor):
        if W.dim() != 3 or W.shape[0] != self.R.ncols:
            raise ValueError(f"W must be {self.R.ncols} matrices, got {tuple(W.shape)}")
        if W.dtype != like.dtype or W.device != like.device:
            raise TypeError("W must have the rows' type and device")
        W = _operand(W)
        return W, W.stride(0) if W.shape[0] > 1 else W.shape[1] * _ld8(W)

    def matmul(self, xs: torch.Tensor, W: torch.Tensor, stream=None) -> torch.Tensor:
        """ys[s] = W[e] xs[s] for the rows s of every column e: xs nnz x K in slot order, W E x N x K, bfloat16 or
        float16; products and sums in 32 bits, rounded once.  Rows behind the placed entries are left unwritten."""
        dt = _dtype(xs, "xs")
        with _on(stream, xs, W):
            xs = _operand(_matrix(xs, "xs", self.nnz))
            W, apart = self._experts(W, xs)
            (_, N, K), Z = W.shape, self.nnz
            if xs.shape[1] != K:
                raise ValueError(f"rows of {xs.shape[1]} values do not fit matrices of {K} columns")
            out = torch.empty((Z, N), dtype=xs.dtype, device=xs.device)
            _abi.ws_routing_matmul(self._r, xs.data_ptr(), _ld8(xs), W.data_ptr(), _ld8(W), apart, N, K,
                                   out.data_ptr(), N, dt, self._queue())
        return out

    def matmul_backward(self, grad_ys: torch.Tensor, xs: torch.Tensor, W: torch.Tensor, stream=None):
        """Gradients of xs (W[e]^T grad_ys[s]) and of W (sum over the rows of e of grad_ys[s] xs[s]^T; zero for a
        column without entries), in their types."""
        dt = _dtype(xs, "xs")
        with _on(stream, grad_ys, xs, W):
            xs = _operand(_matrix(xs, "xs", self.nnz))
            g = _operand(_matrix(grad_ys, "grad_ys", self.nnz, xs))
            W, apart = self._experts(W, xs)
            (E, N, K), Z, raw = W.shape, self.nnz, self._queue()
            if xs.shape[1] != K or g.shape[1] != N:
                raise ValueError(f"rows of {xs.shape[1]} and {g.shape[1]} values do not fit matrices {N} x {K}")
            gxs = torch.empty((Z, K), dtype=xs.dtype, device=xs.device)
            gW = torch.empty((E, N, K), dtype=xs.dtype, device=xs.device)
            _abi.ws_routing_matmul_rows(self._r, g.data_ptr(), _ld8(g), W.data_ptr(), _ld8(W), apart, N, K,
                                        gxs.data_ptr(), K, dt, raw)
            _abi.ws_routing_matmul_weights(self._r, g.data_ptr(), _ld8(g), xs.data_ptr(), _ld8(xs), N, K,
                                           gW.data_ptr(), K, N * K, dt, raw)
        return gxs, gW

    def wait(self, stream=None) -> None:
        """Waits for the stream and raises if a product's kernel gave up a wait since the plan was built."""
        with _on(stream):
            self._queue()
            torch.cuda.current_stream(self.device).synchronize()
        at = 2 * (self.R.ncols + 1) + 3 * self.nnz
        if int(self._buf[at]):
            raise _abi.WsError("Routing.wait", 8, "a product's kernel gave up a wait")


def adapters(x: torch.Tensor, A: torch.Tensor, B: torch.Tensor, S: DeviceCSR, base: torch.Tensor | None = None,
             out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """y[t] = base[t] + sum over row t of S of value * B[a] (A[a] x[t]): low-rank adapters of many requests beside the
    projection they share (``base``, its result; None for zero).

    x: T x K, A: L x r x K, B: L x N x r, base: T x N, bfloat16 or float16; S: T x L in CSR, float32 values, rows empty
    for tokens without an adapter.  ``out`` may be ``base``: the adapters' part is then added in place.
    """
    dt = _dtype(x, "x")
    if A.dim() != 3 or B.dim() != 3 or A.shape[0] != B.shape[0] or A.shape[1] != B.shape[2]:
        raise ValueError(f"A must be L x r x K and B L x N x r, got {tuple(A.shape)} and {tuple(B.shape)}")
    (L, r, K), N, T = A.shape, B.shape[1], S.nrows
    if A.dtype != x.dtype or B.dtype != x.dtype or A.device != x.device or B.device != x.device:
        raise TypeError("x, A and B must have one type and device")
    for t, d in ((S.rowptr, torch.int64), (S.colidx, torch.int32), (S.vals, torch.float32)):
        if t.dtype != d or t.device != x.device or not t.is_contiguous():
            raise TypeError("S must hold contiguous int64/int32/float32 tensors on x's device")
    nnz = S.colidx.numel()
    if S.ncols != L or S.rowptr.numel() != T + 1 or S.vals.numel() != nnz:
        raise ValueError(f"S must be {x.shape[0]} x {L} in CSR")
    with _on(stream, x, A, B, S.rowptr, S.colidx, S.vals, *(() if base is None else (base,))):
        x = _operand(_matrix(x, "x", T))
        if x.shape[1] != K:
            raise ValueError(f"rows of {x.shape[1]} values do not fit adapters of {K}")
        A = _operand(A)
        if (r > 1 and B.stride(2) != 1) or (N > 1 and B.stride(1) < r):
            B = B.contiguous()
        if base is not None:
            base = _matrix(base, "base", T, x)
            if base.shape[1] != N:
                raise ValueError(f"base must be {T} x {N}")
        if out is None:
            out = torch.empty((T, N), dtype=x.dtype, device=x.device)
        elif _matrix(out, "out", T, x) is not out or out.shape[1] != N:
            raise ValueError(f"out must be {T} x {N} with unit stride within its rows")
        elif base is not None and _overlap(out, base) and (out.data_ptr(), _ld(out)) != (base.data_ptr(), _ld(base)):
            raise ValueError("out must be base itself or lie apart from it")
        need = _abi.ws_adapters_scratch(nnz, r)
        scratch = torch.empty(need, dtype=torch.uint8, device=x.device)
        call = _abi.WsAdaptersCall(T, L, nnz, S.rowptr.data_ptr(), S.colidx.data_ptr(), S.vals.data_ptr(), K, r, N,
                                   x.data_ptr(), _ld8(x), A.data_ptr(), _ld8(A), A.stride(0), B.data_ptr(),
                                   B.stride(1), B.stride(0), 0 if base is None else base.data_ptr(),
                                   0 if base is None else _ld(base), out.data_ptr(), _ld(out), dt)
        _abi.ws_adapters(call, scratch.data_ptr(), need, _raw_stream(x.device))
    return out


def _overlap(a: torch.Tensor, b: torch.Tensor) -> bool:
    """Whether the address ranges of two matrices meet."""
    def span(t):
        if t.numel() == 0:
            return t.data_ptr(), t.data_ptr()
        return t.data_ptr(), t.data_ptr() + ((t.shape[0] - 1) * t.stride(0) + t.shape[1]) * t.element_size()
    (a0, a1), (b0, b1) = span(a), span(b)
    return a0 < b1 and b0 < a1
