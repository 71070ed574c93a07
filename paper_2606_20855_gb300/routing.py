"""Operations on sparse routing matrices: rows of dense matrices sent along a CSR matrix.

A routing matrix R (:class:`DeviceCSR`, float32 values, at most 1024 columns) has a row per token and a column per
expert.  A layer of experts is

    R = topk_route(logits, k)          # k experts of every token and their weights
    plan = Routing(R)                  # R transposed: the tokens sorted by expert
    xs = plan.dispatch(x)              # their rows in that order
    y = plan.combine(f(xs))            # the experts' rows summed back with R's values

where the experts' matrices may be ``plan.matmul(xs, W)``; the gradients are ``combine_backward``,
``dispatch_backward``, ``matmul_backward`` and ``topk_route_backward``.  All calls queue work on
the current stream, or on ``stream``, and return without waiting; none reads anything back.  Tensors are on the current
device.
"""
from __future__ import annotations

import ctypes
import functools

import torch

from . import _abi
from .spgemm import DeviceCSR

_ROW_DTYPES = {torch.float32: _abi.WS_F32, torch.bfloat16: _abi.WS_BF16, torch.float16: _abi.WS_F16}
_raw_stream = torch._C._cuda_getCurrentRawStream  # of a device, without building the object
_current_device = torch._C._cuda_getDevice


def _queue_of(index: int) -> int:
    """The current stream of the tensors' device, which has to be the current device: the library launches there."""
    if _current_device() != index:
        raise ValueError(f"tensors on device {index}, but device {_current_device()} is current")
    return _raw_stream(index)


def _elsewhere(f, stream, *args, **kwargs):
    """f on ``stream``: results are allocated and work is queued there; inputs that came from another stream stay
    allocated until it is done with them."""
    for t in (*args, *kwargs.values()):
        for u in (t.rowptr, t.colidx, t.vals) if isinstance(t, DeviceCSR) else (t,):
            if isinstance(u, torch.Tensor):
                u.record_stream(stream)
    with torch.cuda.stream(stream):
        return f(*args, **kwargs)


def _dtype(t: torch.Tensor, name: str) -> int:
    dt = _ROW_DTYPES.get(t.dtype)
    if dt is None:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    if not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    return dt


def _same(t: torch.Tensor, like: torch.Tensor, name: str) -> None:
    if t.dtype != like.dtype or t.device != like.device:
        raise TypeError(f"{name} must have the other matrix's type and device")


def _matrix(t: torch.Tensor, name: str, rows: int | None):
    """(t, its row stride): a 2-D tensor whose rows have unit stride (copied if they have not)."""
    if t.dim() != 2 or (rows is not None and t.shape[0] != rows):
        raise ValueError(f"{name} must be 2-D" + (f" with {rows} rows" if rows is not None else "") +
                         f", got {tuple(t.shape)}")
    n = t.shape[1]
    if t.is_contiguous():
        return t, n
    if (n > 1 and t.stride(1) != 1) or (t.shape[0] > 1 and t.stride(0) < n):
        return t.contiguous(), n
    return t, t.stride(0) if t.shape[0] > 1 else n


def _operand(t: torch.Tensor):
    """(t, its row stride, that of a stack's matrices, bytes of a copy): a matrix or a stack of matrices of 16-bit
    values with unit stride within a row.  The copy is made by the call where rows do not start at multiples of 16
    bytes."""
    shape = t.shape
    n, rows = shape[-1], shape[-2]
    if t.is_contiguous():
        if n % 8 == 0 and t.data_ptr() % 16 == 0:
            return t, n, n * rows, 0
        return t, n, n * rows, t.numel() // max(n, 1) * ((n + 7) // 8 * 16)
    if n > 1 and t.stride(-1) != 1:
        return _operand(t.contiguous())
    ld = t.stride(-2)
    apart = t.stride(0) if t.dim() == 3 else 0
    if t.data_ptr() % 16 == 0 and (rows <= 1 or (ld % 8 == 0 and ld >= n)) and \
            (t.dim() == 2 or shape[0] <= 1 or apart % 8 == 0):
        return t, ld, apart, 0
    return t, ld, apart, t.numel() // max(n, 1) * ((n + 7) // 8 * 16)


def _room(need: int, device):
    """(tensor, address) of scratch; (None, 0) where none is needed."""
    if need == 0:
        return None, 0
    t = torch.empty(need, dtype=torch.uint8, device=device)
    return t, t.data_ptr()


def topk_route(logits: torch.Tensor, k: int, normalize: bool = True, stream=None) -> DeviceCSR:
    """The routing matrix of a T x E tensor of logits: row i holds the k largest logits of row i (ties to the lowest
    column), by ascending column, with softmax weights over the chosen (``normalize``) or over all columns.  A logit
    of -inf has weight 0 and is chosen last; a row of nothing else has weights 0."""
    if stream is not None:
        return _elsewhere(topk_route, stream, logits, k, normalize)
    dt = _dtype(logits, "logits")
    x, ld = _matrix(logits, "logits", None)
    (T, E), k, dev = x.shape, int(k), x.device
    if k < 1 or k > E or k > 32:
        raise ValueError(f"k must be in 1..min(columns, 32), got {k} of {E}")
    rowptr = torch.empty(T + 1, dtype=torch.int64, device=dev)
    colidx = torch.empty(T * k, dtype=torch.int32, device=dev)
    vals = torch.empty(T * k, dtype=torch.float32, device=dev)
    _abi.ws_topk_route(x.data_ptr(), T, E, ld, dt, k, normalize, rowptr.data_ptr(), colidx.data_ptr(), vals.data_ptr(),
                       _queue_of(dev.index))
    return DeviceCSR(T, E, rowptr, colidx, vals)


def topk_route_backward(logits: torch.Tensor, R: DeviceCSR, grad_vals: torch.Tensor, normalize: bool = True,
                        stream=None) -> torch.Tensor:
    """Gradient of the logits from that of R's values, for ``R = topk_route(logits, k, normalize)``."""
    if stream is not None:
        return _elsewhere(topk_route_backward, stream, logits, R, grad_vals, normalize)
    dt = _dtype(logits, "logits")
    x, ld = _matrix(logits, "logits", R.nrows)
    T, E = x.shape
    nnz = R.colidx.numel()
    k = nnz // T if T else 1
    if E != R.ncols or k * T != nnz:
        raise ValueError("R is not the routing matrix of these logits")
    vals = R.vals
    if grad_vals.dtype != torch.float32 or grad_vals.numel() != nnz or vals.dtype != torch.float32:
        raise TypeError("grad_vals must be float32, one for every value of R")
    if grad_vals.device != x.device or R.colidx.dtype != torch.int32 or R.colidx.device != x.device:
        raise TypeError("R and grad_vals must be on the logits' device")
    g, vals, cols = grad_vals.contiguous(), vals.contiguous(), R.colidx.contiguous()
    out = torch.empty((T, E), dtype=x.dtype, device=x.device)
    _abi.ws_topk_route_backward(x.data_ptr(), T, E, ld, dt, k, normalize, cols.data_ptr(), vals.data_ptr(),
                                g.data_ptr(), out.data_ptr(), E, _queue_of(x.device.index))
    return out


@functools.lru_cache(maxsize=256)
def _scratch(nrows: int, ncols: int, device: int) -> int:
    return _abi.ws_routing_scratch(nrows, ncols)


@functools.lru_cache(maxsize=1024)
def _adapters_scratch(nnz: int, r: int) -> int:
    return _abi.ws_adapters_scratch(nnz, r)


@functools.lru_cache(maxsize=1024)
def _adapters_many(nrows: int, r: int) -> bool:
    return _abi.ws_adapters_many(nrows, r)


class Routing:
    """A routing matrix with its transpose: the entries of R sorted by column, rows in order within a column.

    ``offsets`` (int64 [E + 1]) is the first slot of every column, ``rows`` and ``entries`` (int32 [nnz]) are the row
    and the entry of R in every slot, ``slots`` (int32 [nnz]) is the slot of every entry.  Entries whose column is out
    of range, or that no row holds (before rowptr[0], from rowptr[T] on), have slot -1 and
    take no part; the slots they leave over come last, hold -1 and stand for zero rows.
    The plan is that of R's shape, row pointer and columns when it is built, and keeps those arrays.  ``combine`` and its
    gradient read R's values as they are at the call, of the tensor that ``R.vals`` is then.

    The products' kernels wait for one another with a limit of two seconds.  One that gives up a wait leaves its result
    incomplete and says so only in ``status`` (int32 [1], nonzero then, cleared when the plan is built): read it where
    results are read, or call ``wait``, which waits for the stream and raises.
    """

    def __init__(self, R: DeviceCSR, validate: bool = False, stream=None):
        if stream is not None:
            _elsewhere(self.__init__, stream, R, validate)
            return
        rowptr, colidx, vals = R.rowptr, R.colidx, R.vals
        if vals.dtype != torch.float32:
            raise TypeError(f"a routing matrix has float32 values, got {vals.dtype}")
        if rowptr.dtype != torch.int64 or colidx.dtype != torch.int32 or rowptr.get_device() < 0 or \
                not rowptr.get_device() == colidx.get_device() == vals.get_device() or \
                not (rowptr.is_contiguous() and colidx.is_contiguous() and vals.is_contiguous()):
            raise TypeError("rowptr/colidx/vals must be contiguous int64/int32/float32 tensors on one GPU")
        self._nrows, self._ncols = T, E = R.nrows, R.ncols
        nnz = colidx.numel()
        if rowptr.numel() != T + 1 or vals.numel() != nnz:
            raise ValueError("rowptr must have nrows + 1 entries, and every column index a value")
        self.R, self.nnz, self.device = R, nnz, rowptr.device
        self._arrays, self._vals = (rowptr, colidx), vals  # whose addresses the calls get
        self._index = self.device.index
        self._stream = raw = _queue_of(self._index)
        if validate:
            _abi.ws_csr_destroy(R._handle(True, raw))
        scratch = _scratch(T, E, self._index)
        # one array: offsets, the status word, the scratch (at a multiple of 16 bytes); rows, entries and slots
        words = (E + 3) // 2 * 2
        self._lead = lead = words + scratch // 8
        self._buf = torch.empty(2 * lead + 3 * nnz, dtype=torch.int32, device=self.device)
        at = self._buf.data_ptr()
        ints = at + 8 * lead
        self._c = _abi.WsRouting(T, E, nnz, rowptr.data_ptr(), colidx.data_ptr(), vals.data_ptr(), at, ints,
                                 ints + 4 * nnz, ints + 8 * nnz, at + 8 * (E + 1))
        self._r = ctypes.byref(self._c)
        _abi.ws_routing_build(self._r, at + 8 * words, scratch, raw)

    def _part(self, first: int, count: int) -> torch.Tensor:
        return self._buf.as_strided((count,), (1,), first)  # the cheapest view on the host

    @property
    def offsets(self) -> torch.Tensor:
        return self._part(0, 2 * self._ncols + 2).view(torch.int64)

    @property
    def rows(self) -> torch.Tensor:
        return self._part(2 * self._lead, self.nnz)

    @property
    def entries(self) -> torch.Tensor:
        return self._part(2 * self._lead + self.nnz, self.nnz)

    @property
    def slots(self) -> torch.Tensor:
        return self._part(2 * self._lead + 2 * self.nnz, self.nnz)

    @property
    def status(self) -> torch.Tensor:
        return self._part(2 * (self._ncols + 1), 1)

    def _rows_of(self, t: torch.Tensor, rows: int, name: str):
        """(t, its row stride, the length of its rows, their type), t being `rows` rows on the plan's device."""
        dt, shape = _ROW_DTYPES.get(t.dtype), t.shape
        if dt is None or len(shape) != 2 or shape[0] != rows or t.get_device() != self._index or not t.is_contiguous():
            dt = _dtype(t, name)
            t, ld = _matrix(t, name, rows)
            if t.get_device() != self._index:
                raise TypeError("the rows and the routing matrix must be on one device")
            return t, ld, shape[1], dt
        return t, shape[1], shape[1], dt

    def _queue(self) -> int:
        """The current stream, for a call; the plan's arrays stay allocated until it is done with them."""
        raw = _queue_of(self._index)
        if raw != self._stream:
            s = torch.cuda.current_stream(self.device)
            for u in (self._buf, *self._arrays, self._vals):
                u.record_stream(s)
        return raw

    def _read_values(self) -> None:
        """R's values for a call that reads them: the tensor may be another one than at the last call."""
        vals = self.R.vals
        if vals is not self._vals:
            if vals.dtype != torch.float32 or vals.get_device() != self._index or not vals.is_contiguous():
                raise TypeError("R's values must be a contiguous float32 tensor on the routing matrix's device")
            if vals.numel() != self.nnz:
                raise ValueError(f"R must have {self.nnz} values, got {vals.numel()}")
            self._vals, self._c.vals = vals, vals.data_ptr()
            vals.record_stream(torch.cuda.current_stream(self.device))

    def dispatch(self, x: torch.Tensor, stream=None) -> torch.Tensor:
        """xs[slot] = x[row]: the rows of x (T x H) in slot order (nnz x H)."""
        if stream is not None:
            return _elsewhere(self.dispatch, stream, x)
        x, ld, H, dt = self._rows_of(x, self._nrows, "x")
        out = torch.empty((self.nnz, H), dtype=x.dtype, device=self.device)
        _abi.ws_routing_dispatch(self._r, x.data_ptr(), ld, out.data_ptr(), H, H, dt, self._queue())
        return out

    def dispatch_backward(self, grad_xs: torch.Tensor, stream=None) -> torch.Tensor:
        """Gradient of x: gx[i] = sum of grad_xs over the slots of row i."""
        if stream is not None:
            return _elsewhere(self.dispatch_backward, stream, grad_xs)
        g, ld, H, dt = self._rows_of(grad_xs, self.nnz, "grad_xs")
        out = torch.empty((self._nrows, H), dtype=g.dtype, device=self.device)
        _abi.ws_routing_dispatch_backward(self._r, g.data_ptr(), ld, out.data_ptr(), H, H, dt, self._queue())
        return out

    def combine(self, ys: torch.Tensor, stream=None) -> torch.Tensor:
        """y[i] = sum over row i of R's value times ys[slot]."""
        if stream is not None:
            return _elsewhere(self.combine, stream, ys)
        ys, ld, H, dt = self._rows_of(ys, self.nnz, "ys")
        self._read_values()
        out = torch.empty((self._nrows, H), dtype=ys.dtype, device=self.device)
        _abi.ws_routing_combine(self._r, ys.data_ptr(), ld, out.data_ptr(), H, H, dt, self._queue())
        return out

    def combine_backward(self, grad_y: torch.Tensor, ys: torch.Tensor, stream=None):
        """Gradients of ys (value times grad_y's row) and of R's values (the products of grad_y's and ys's rows)."""
        if stream is not None:
            return _elsewhere(self.combine_backward, stream, grad_y, ys)
        ys, ld, H, dt = self._rows_of(ys, self.nnz, "ys")
        g, ldg, same, dtg = self._rows_of(grad_y, self._nrows, "grad_y")
        if dtg != dt:
            raise TypeError("grad_y must have the other matrix's type and device")
        if same != H:
            raise ValueError("grad_y and ys differ in the length of their rows")
        self._read_values()
        out = torch.empty((self.nnz, H), dtype=ys.dtype, device=self.device)
        gvals = torch.empty(self.nnz, dtype=torch.float32, device=self.device)
        _abi.ws_routing_combine_backward(self._r, g.data_ptr(), ldg, ys.data_ptr(), ld, out.data_ptr(), H,
                                         gvals.data_ptr(), H, dt, self._queue())
        return out, gvals

    def _product(self, xs: torch.Tensor, W: torch.Tensor):
        """(type, N, K) of a product."""
        dt, stack, rows = _dtype(xs, "xs"), W.shape, xs.shape
        if len(stack) != 3 or stack[0] != self._ncols:
            raise ValueError(f"W must be {self._ncols} matrices, got {tuple(stack)}")
        if W.dtype != xs.dtype or not W.get_device() == xs.get_device() == self._index:
            raise TypeError("W and xs must have one type and be on the routing matrix's device")
        _, N, K = stack
        if len(rows) != 2 or rows[0] != self.nnz or rows[1] != K:
            raise ValueError(f"xs must be {self.nnz} rows of {K} values, got {tuple(rows)}")
        return dt, N, K

    def matmul(self, xs: torch.Tensor, W: torch.Tensor, stream=None) -> torch.Tensor:
        """ys[s] = W[e] xs[s] for the rows s of every column e: xs nnz x K in slot order, W E x N x K, bfloat16 or
        float16; products and sums in 32 bits, rounded once.  Rows behind the placed entries are zero."""
        if stream is not None:
            return _elsewhere(self.matmul, stream, xs, W)
        dt, N, K = self._product(xs, W)
        xs, ldx, _, a = _operand(xs)
        W, ldw, apart, b = _operand(W)
        out = torch.empty((self.nnz, N), dtype=xs.dtype, device=self.device)
        room, at = _room(a + b, self.device)
        _abi.ws_routing_matmul(self._r, xs.data_ptr(), ldx, W.data_ptr(), ldw, apart, N, K, out.data_ptr(), N, dt, at,
                               a + b, self._queue())
        return out

    def matmul_backward(self, grad_ys: torch.Tensor, xs: torch.Tensor, W: torch.Tensor, stream=None):
        """Gradients of xs (W[e]^T grad_ys[s]) and of W (sum over the rows of e of grad_ys[s] xs[s]^T; zero for a
        column without entries), in their types."""
        if stream is not None:
            return _elsewhere(self.matmul_backward, stream, grad_ys, xs, W)
        (dt, N, K), E = self._product(xs, W), self._ncols
        _same(grad_ys, xs, "grad_ys")
        if grad_ys.dim() != 2 or grad_ys.shape[0] != self.nnz or grad_ys.shape[1] != N:
            raise ValueError(f"grad_ys must be {self.nnz} rows of {N} values, got {tuple(grad_ys.shape)}")
        g, ldg, _, a = _operand(grad_ys)
        xs, ldx, _, b = _operand(xs)
        W, ldw, apart, c = _operand(W)
        gxs = torch.empty((self.nnz, K), dtype=xs.dtype, device=self.device)
        gW = torch.empty((E, N, K), dtype=xs.dtype, device=self.device)
        room, at = _room(a + b + c, self.device)
        _abi.ws_routing_matmul_backward(self._r, g.data_ptr(), ldg, xs.data_ptr(), ldx, W.data_ptr(), ldw, apart, N, K,
                                        gxs.data_ptr(), K, gW.data_ptr(), K, N * K, dt, at, a + b + c, self._queue())
        return gxs, gW

    def wait(self, stream=None) -> None:
        """Waits for the stream and raises if a product's kernel gave up a wait since the plan was built."""
        if stream is not None:
            return _elsewhere(self.wait, stream)
        self._queue()
        torch.cuda.current_stream(self.device).synchronize()
        if int(self.status):
            raise _abi.WsError("Routing.wait", 8, "a product's kernel gave up a wait")


def adapters(x: torch.Tensor, A: torch.Tensor, B: torch.Tensor, S: DeviceCSR, base: torch.Tensor | None = None,
             out: torch.Tensor | None = None, stream=None, wait: bool = False,
             status: torch.Tensor | None = None) -> torch.Tensor:
    """y[t] = base[t] + sum over row t of S of value * B[a] (A[a] x[t]): low-rank adapters of many requests beside the
    projection they share (``base``, its result; None for zero).

    x: T x K, A: L x r x K, B: L x N x r, base: T x N, bfloat16 or float16; S: T x L in CSR, float32 values, rows empty
    for tokens without an adapter.  ``out`` may be ``base``: the adapters' part is then added in place; it may overlap no
    other input.

    The kernels for many tokens wait for one another with a limit of two seconds.  One that gives up a wait leaves y
    incomplete.  ``status`` (int32, one value, of the caller's) is then made nonzero, and left as it is otherwise, so that one
    serves many calls; ``wait`` waits for the result and raises.
    """
    if stream is not None:
        return _elsewhere(adapters, stream, x, A, B, S, base, out, wait=wait, status=status)
    dt, dtype, dev, index = _dtype(x, "x"), x.dtype, x.device, x.get_device()
    (La, r, K), (L, N, rb) = A.shape, B.shape
    if La != L or r != rb:
        raise ValueError(f"A must be L x r x K and B L x N x r, got {tuple(A.shape)} and {tuple(B.shape)}")
    if not A.dtype == B.dtype == dtype or not A.get_device() == B.get_device() == index:
        raise TypeError("A and B must have x's type and device")
    rowptr, colidx, vals, T, rows = S.rowptr, S.colidx, S.vals, S.nrows, x.shape
    if rowptr.dtype != torch.int64 or colidx.dtype != torch.int32 or vals.dtype != torch.float32 or \
            not (rowptr.is_contiguous() and colidx.is_contiguous() and vals.is_contiguous()) or \
            not rowptr.get_device() == colidx.get_device() == vals.get_device() == index:
        raise TypeError("S must hold contiguous int64/int32/float32 tensors on x's device")
    nnz = colidx.numel()
    if S.ncols != L or rowptr.numel() != T + 1 or vals.numel() != nnz:
        raise ValueError(f"S must be {rows[0]} x {L} in CSR")
    if len(rows) != 2 or rows[0] != T or rows[1] != K:
        raise ValueError(f"x must be {T} rows of {K} values, got {tuple(rows)}")
    x, ldx, _, need = _operand(x)
    A, lda, apart, more = _operand(A)
    B, ldb, apartB, most = _operand(B)
    if status is not None and (status.dtype != torch.int32 or status.numel() != 1 or status.get_device() != index):
        raise TypeError("status must be one int32 value on x's device")
    many = _adapters_many(T, r) and N > 0
    need = _adapters_scratch(nnz, r) + (need + more + most if many else 0)
    ldbase = ldy = N
    if base is not None:
        if base.dtype != dtype or base.get_device() != index:
            raise TypeError("base must have x's type and device")
        base, ldbase = _matrix(base, "base", T)
        if base.shape[1] != N:
            raise ValueError(f"base must be {T} x {N}")
    if out is None:
        out = torch.empty((T, N), dtype=dtype, device=dev)
    else:
        _same(out, x, "out")
        same, ldy = _matrix(out, "out", T)
        if same is not out or out.shape[1] != N:
            raise ValueError(f"out must be {T} x {N} with unit stride within its rows")
        if base is not None and (out.data_ptr(), ldy) != (base.data_ptr(), ldbase) and _overlap(out, base):
            raise ValueError("out must be base itself or lie apart from it")
        first, end = _span(out)
        for t, name in ((x, "x"), (A, "A"), (B, "B"), (rowptr, "S"), (colidx, "S"), (vals, "S")):
            a, b = _span(t)
            if a < end and first < b and _overlap(out, t):  # it is written while they are read
                raise ValueError(f"out must lie apart from {name}")
    scratch = torch.empty(need, dtype=torch.uint8, device=dev)
    call = _abi.ADAPTERS_CALL.pack(T, L, nnz, rowptr.data_ptr(), colidx.data_ptr(), vals.data_ptr(), K, r, N,
                                   x.data_ptr(), ldx, A.data_ptr(), lda, apart, B.data_ptr(), ldb, apartB,
                                   0 if base is None else base.data_ptr(), ldbase, out.data_ptr(), ldy, dt)
    _abi.ws_adapters(call, scratch.data_ptr(), need, _queue_of(index))
    if many and status is not None:
        status.bitwise_or_(scratch[:4].view(torch.int32).view(status.shape))
    if wait:
        torch.cuda.current_stream(dev).synchronize()
        if many and scratch[:4].view(torch.int32).item():
            raise _abi.WsError("adapters", 8, "a kernel gave up a wait")
    return out


def _span(t: torch.Tensor):
    """First address of a tensor and the one behind its last."""
    at = t.data_ptr()
    if t.is_contiguous():
        return at, at + t.nbytes
    return at, at + (sum((n - 1) * s for n, s in zip(t.shape, t.stride())) + 1) * t.element_size()


def _overlap(a: torch.Tensor, b: torch.Tensor) -> bool:
    """Whether two tensors, of unit stride within a row, may share memory: their address ranges meet, and neither's rows
    all lie between the other's (as column blocks of one matrix do)."""
    if a.numel() == 0 or b.numel() == 0:
        return False

    def row(t):  # bytes of a row
        return (t.shape[-1] - 1) * t.stride(-1) * t.element_size() + t.element_size()

    def steps(t):  # bytes from row to row and from matrix to matrix
        return [t.stride(i) * t.element_size() for i in range(t.dim() - 1) if t.shape[i] > 1]

    def between(inner, outer):
        if outer.dim() != 2 or outer.shape[0] < 2:
            return False
        ld = outer.stride(0) * outer.element_size()
        at = (inner.data_ptr() - outer.data_ptr()) % ld
        return at >= row(outer) and at + row(inner) <= ld and all(s % ld == 0 for s in steps(inner))

    (a0, a1), (b0, b1) = _span(a), _span(b)
    return a0 < b1 and b0 < a1 and not between(a, b) and not between(b, a)
