"""The optimizer of a layer's weights: one launch of AdamW over many tensors.

    opt = AdamW([w.master for w in weights], copies=[w.half for w in weights])
    opt.step(grads)        # masters, states and 16-bit copies are updated in place

Work is queued on the current stream, or on ``stream``; nothing is read back, so that a step can be captured in a graph.
"""
from __future__ import annotations

import ctypes
import struct

import torch

from . import _abi
from .routing import _ROW_DTYPES, _queue_of, _span

# of every gradient in turn: to call the methods themselves takes the host less
_numel, _contiguous, _place, _address = torch.Tensor.numel, torch.Tensor.is_contiguous, torch.Tensor.get_device, torch.Tensor.data_ptr
_written_to = torch._C._increment_version  # of a list of tensors, as torch.autograd.graph.increment_version

BLOCK = 256  # values that share a scale where states have 8 bits


class AdamW:
    """AdamW over ``params``, contiguous float32 tensors on one device.  For every value, t being the number of the step, one count for all
    tensors (also for one that has had no gradient until now: its first change is then up to (1 - b1) / sqrt(1 - b2) lr, 3.2 lr with
    the default betas, where a count of its own would make it lr; a gradient of zeros counts as one):

        m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2
        p = p (1 - lr weight_decay) - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps)

    lr: a number, or a float32 tensor of one value on the device (read when a step runs, also in a captured graph); it may be
    replaced between steps.  weight_decay: a number, or one for every tensor.  eps: 0, or at least 2^-126.
    copies: bfloat16 or float16 tensors of the parameters' sizes (or None), which get the new values rounded.
    bits: 32, m and v are float32; or 8, m and sqrt(v) are float8_e4m3fn codes with a float32 scale for every 256 values of a
    tensor, rounded stochastically by a hash of seed, step, tensor and place (equal inputs give equal bits); eps is at least 1e-15
    then, as roots below 2^-63 count as 0.
    state: that of another optimizer, used and updated as it is, not copied: the dict that ``state`` is.  Its entries are lists of
    a tensor for every parameter, "m" and "v", or "m", "r", "m_scale" and "r_scale", and "step", int64 [1], steps done.

    A step counts as an operation in place on the parameters and copies that it updates: a backward pass that needs their old values is an
    error, as with any operation of torch (but not where a captured step is replayed).

    No two steps of one optimizer, or of two that share tensors, may run at the same time.
    """

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay=0.01, bits: int = 32, copies=None,
                 seed: int = 0, state: dict | None = None):
        params = list(params)
        if not params:
            raise ValueError("no parameters")
        if bits not in (8, 32):
            raise ValueError(f"states have 8 or 32 bits, got {bits}")
        beta1, beta2 = (float(b) for b in betas)
        if not (0 <= beta1 < 1 and 0 <= beta2 < 1 and eps >= 0):
            raise ValueError(f"betas must be in [0, 1) and eps not negative, got {betas} and {eps}")
        if 0 < eps < 2.0 ** -126:
            raise ValueError(f"eps must be 0 or a normal number of 32 bits, got {eps}")
        if bits == 8 and eps < 1e-15:
            raise ValueError(f"with states of 8 bits eps must be at least 1e-15, got {eps}")
        self.device, self._index = params[0].device, params[0].get_device()
        if self._index < 0:
            raise TypeError("params must be CUDA tensors")
        self._seen = {_queue_of(self._index)}  # streams on which the tensors were used
        for p in params:
            self._tensor(p, torch.float32, p.numel(), "params")
        self.params, self.bits, self.seed = params, bits, int(seed) & 0xFFFFFFFF
        self.betas, self.eps, self.lr = (beta1, beta2), float(eps), lr
        sizes = self._sizes = [p.numel() for p in params]
        count = len(params)
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * count
        copies = [None] * count if copies is None else list(copies)
        if len(decay) != count or len(copies) != count:
            raise ValueError(f"weight_decay and copies must have an entry for each of {count} tensors")
        types = {c.dtype for c in copies if c is not None}
        if len(types) > 1 or not types <= {torch.bfloat16, torch.float16}:
            raise TypeError(f"copies must be bfloat16 or float16, all the same, got {types}")
        for c, n in zip(copies, sizes):
            if c is not None:
                self._tensor(c, c.dtype, n, "copies")
        self.copies = copies
        blocks = [-(-n // BLOCK) for n in sizes]
        if bits == 32:
            kinds = {"m": (torch.float32, sizes), "v": (torch.float32, sizes)}
        else:
            f8 = torch.float8_e4m3fn
            kinds = {"m": (f8, sizes), "r": (f8, sizes), "m_scale": (torch.float32, blocks), "r_scale": (torch.float32, blocks)}
        if state is None:
            state = {name: [torch.zeros(n, dtype=torch.uint8 if bits == 8 and dt != torch.float32 else dt, device=self.device).view(dt)
                            for n in lengths] for name, (dt, lengths) in kinds.items()}
            state["step"] = torch.zeros(1, dtype=torch.int64, device=self.device)
        if set(state) != {*kinds, "step"}:
            raise ValueError(f"state must have {', '.join(kinds)} and step, got {', '.join(state)}")
        for name, (dt, lengths) in kinds.items():
            if len(state[name]) != count:
                raise ValueError(f"state[{name!r}] must have {count} tensors")
            for t, n in zip(state[name], lengths):
                self._tensor(t, dt, n, f"state[{name!r}]")
        self._tensor(state["step"], torch.int64, 1, "state['step']")
        self.state = state
        self._apart([*params, *(c for c in copies if c is not None), *(t for name in kinds for t in state[name]), state["step"]])
        self._done = torch.zeros(1, dtype=torch.int32, device=self.device)  # the kernel's own count, 0 between steps
        self._copy_type = _ROW_DTYPES[types.pop()] if types else _abi.WS_BF16
        second = "v" if bits == 32 else "r"
        table = bytearray()
        for i, p in enumerate(params):
            scales = (state["m_scale"][i].data_ptr(), state["r_scale"][i].data_ptr()) if bits == 8 else (0, 0)
            table += _abi.ADAMW_TENSOR.pack(p.data_ptr(), state["m"][i].data_ptr(), state[second][i].data_ptr(), *scales,
                                            0 if copies[i] is None else copies[i].data_ptr(), sizes[i], float(decay[i]))
        self._table = ctypes.create_string_buffer(bytes(table), len(table))
        self._at_table, self._at_step, self._at_done = ctypes.addressof(self._table), state["step"].data_ptr(), self._done.data_ptr()
        self._pointers, self._pack = (ctypes.c_void_p * count)(), struct.Struct(f"={count}Q")
        self._at_pointers = ctypes.addressof(self._pointers)
        self._written = [t for t in (*params, *copies) if t is not None]  # what a backward pass may need as it was

    def _one(self, t: torch.Tensor, dtype, name: str) -> int:
        if t.dtype != dtype or t.numel() != 1 or t.get_device() != self._index:
            raise TypeError(f"{name} must be one {dtype} value on the parameters' device")
        return t.data_ptr()

    def step(self, grads, scale: torch.Tensor | None = None, skip: torch.Tensor | None = None, stream=None) -> None:
        """One step.  grads: a tensor of its size for every parameter, all float32, bfloat16 or float16, apart from what
        the step writes; None: that parameter stays as it is.  Gradients are multiplied by ``scale`` (float32, one value on the
        device) first; where ``skip`` (int32, one value) is not 0 the step does nothing and is not counted."""
        if stream is not None:
            for t in (*grads, scale, skip, self.lr):
                if isinstance(t, torch.Tensor) and t.is_cuda:
                    t.record_stream(stream)
            with torch.cuda.stream(stream):
                return self.step(grads, scale, skip)
        if len(grads) != len(self._sizes):
            raise ValueError(f"{len(grads)} gradients for {len(self._sizes)} parameters")
        raw = _queue_of(self._index)
        if raw not in self._seen:
            self._record(raw)
        held = None  # copies, until the launch has been queued
        try:  # the usual: all of them, as they are
            usual = [*map(_numel, grads)] == self._sizes and all(map(_contiguous, grads))
        except TypeError:  # None among them
            usual = False
        if usual:
            kinds, places = {g.dtype for g in grads}, set(map(_place, grads))
            at, written = [*map(_address, grads)], self._written
        else:
            held = [g if g is None or g.is_contiguous() else g.contiguous() for g in grads]
            kinds, places = {g.dtype for g in held if g is not None}, {g.get_device() for g in held if g is not None}
            at = [0 if g is None else g.data_ptr() for g in held]
            for i, (g, n) in enumerate(zip(held, self._sizes)):
                if g is not None and g.numel() != n:
                    raise ValueError(f"gradient {i} must have the parameter's {n} values, got {tuple(g.shape)}")
            written = [t for g, p, c in zip(grads, self.params, self.copies) if g is not None for t in (p, c) if t is not None]
        if len(kinds) > 1 or not kinds <= _ROW_DTYPES.keys():
            raise TypeError(f"gradients must be float32, bfloat16 or float16, all the same, got {kinds}")
        if places - {self._index}:
            raise ValueError(f"gradients must be on the parameters' device {self.device}")
        self._pack.pack_into(self._pointers, 0, *at)
        kind = kinds.pop() if kinds else None
        lr, at_lr = self.lr, 0
        if isinstance(lr, torch.Tensor):
            lr, at_lr = 0.0, self._one(lr, torch.float32, "lr")
        at_scale = 0 if scale is None else self._one(scale, torch.float32, "scale")
        at_skip = 0 if skip is None else self._one(skip, torch.int32, "skip")
        call = _abi.ADAMW_CALL.pack(self._at_table, self._at_pointers, len(at), self._at_step, self._at_done, at_lr, at_scale, at_skip, lr,
                                    *self.betas, self.eps, self.seed, self.bits, _ROW_DTYPES[kind] if kind is not None else _abi.WS_F32,
                                    self._copy_type)
        _abi.ws_adamw(call, raw)
        _written_to(written)

    def _record(self, raw: int) -> None:
        """The tensors stay allocated until the current stream, a new one, is done with them."""
        s = torch.cuda.current_stream(self.device)
        for t in (*self.params, *self.copies, self._done, self.state["step"], *(t for k, v in self.state.items() if k != "step" for t in v)):
            if t is not None:
                t.record_stream(s)
        self._seen.add(raw)

    def _tensor(self, t, dtype, n, name):
        if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.get_device() != self._index or not t.is_contiguous():
            raise TypeError(f"{name} must hold contiguous {dtype} tensors on one device")
        if t.numel() != n:
            raise ValueError(f"{name} must have as many values as the parameter asks for: {n}, got {t.numel()}")

    @staticmethod
    def _apart(tensors):
        spans = sorted(_span(t) for t in tensors if t.numel())
        for (_, end), (begin, _) in zip(spans, spans[1:]):
            if begin < end:
                raise ValueError("parameters, copies and states must lie apart from one another")
