"""AdamW over many tensors at once (``t2i_op_adamw_step``): takes the gradients that the
``_backward`` calls return to the weights.

Argument marshalling only; the conventions are those of ``ops.py``.
"""
from __future__ import annotations

import ctypes as C
import math
from array import array
from operator import attrgetter, is_
from typing import Iterable, Optional, Sequence, Union

import torch
from torch.autograd import forward_ad

from ._lib import T2I_BF16, T2I_F32, T2IError, load
from .ops import _check, _elsewhere, _need, _stream, _switch

_DTYPES = {torch.bfloat16: T2I_BF16, torch.float32: T2I_F32}


_shape, _dtype, _requires_grad = attrgetter("shape"), attrgetter("dtype"), attrgetter("requires_grad")
_pointer, _device_of, _whole = torch.Tensor.data_ptr, torch.Tensor.get_device, torch.Tensor.is_contiguous
assert array("Q").itemsize == C.sizeof(C.c_void_p)


def _scalar(t: Optional[torch.Tensor], dev: int, what: str):
    """Pointer of a device scalar that a kernel reads, or None"""
    if t is None:
        return None
    if t.dtype is not torch.float32 or t.numel() != 1 or t.get_device() != dev:
        raise T2IError(1, f"{what} must be one fp32 value on the weights' device")
    return t.data_ptr()


class AdamW:
    """AdamW for a fixed list of weights, updated in place by :meth:`step`.

    ``params``: contiguous device tensors of one device and type (bf16 or fp32).  The moments
    are fp32: zeros, or the given ``exp_avg`` and ``exp_avg_sq`` with the number of ``step`` s
    behind them.  bf16 weights have fp32 ``masters`` -- the given ones, or copies -- whose
    rounded values they receive.  All of these are kept (attributes of the same names), to be
    saved and passed in again by a program that resumes.  A weight's storage, or its tensor in
    ``params``, may be exchanged between steps, the moments' and masters' may not.

    With ``capturable`` the number of steps is counted on the device, so that a captured
    :meth:`step` counts on from replay to replay; without it a step is refused while a graph
    is captured."""

    def __init__(self, params: Sequence[torch.Tensor], *, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8,
                 weight_decay: float = 0.01, masters: Optional[Sequence[torch.Tensor]] = None,
                 exp_avg: Optional[Sequence[torch.Tensor]] = None,
                 exp_avg_sq: Optional[Sequence[torch.Tensor]] = None, step: int = 0, capturable: bool = False):
        self.params = list(params)
        _need(len(self.params) > 0, "no weights")
        first = self.params[0]
        if first.dtype not in _DTYPES:
            raise T2IError(1, "weights must be bf16 or fp32")
        self._dev = first.get_device()
        _need(self._dev >= 0, "weights must be device tensors", 1)
        _need(0 <= betas[0] < 1 and 0 <= betas[1] < 1, "betas must be in [0, 1)", 1)
        _need(eps >= 0 and all(map(math.isfinite, (lr, eps, weight_decay))),
              "lr, eps and weight_decay must be finite, eps >= 0", 1)
        _need(step >= 0 and step == int(step), "step must be a whole number, >= 0", 1)
        self.lr, self.betas, self.eps, self.weight_decay = lr, tuple(betas), eps, weight_decay
        self._type = _DTYPES[first.dtype]
        self._shapes = [p.shape for p in self.params]
        self._numel = (C.c_int64 * len(self.params))(*[p.numel() for p in self.params])
        low = self._type == T2I_BF16
        _need(low or masters is None, "masters go with bf16 weights", 1)
        with torch.no_grad():
            if low and masters is None:
                masters = [m.copy_(p) for m, p in zip(self._new(torch.empty), self.params)]
            if exp_avg is None and exp_avg_sq is None:
                _need(step == 0, "steps behind the moments go with moments", 1)
                exp_avg, exp_avg_sq = self._new(torch.zeros), self._new(torch.zeros)
        _need(exp_avg is not None and exp_avg_sq is not None, "exp_avg and exp_avg_sq go together", 1)
        self.masters = None if masters is None else list(masters)
        self.exp_avg, self.exp_avg_sq = list(exp_avg), list(exp_avg_sq)
        self._state = [("params", self.params, first.dtype), ("exp_avg", self.exp_avg, torch.float32),
                       ("exp_avg_sq", self.exp_avg_sq, torch.float32)]
        if low:
            self._state.append(("masters", self.masters, torch.float32))
        self._kept = [t for _, tensors, _ in self._state[1:] for t in tensors]
        self._lay_out()
        _need(not any(t.requires_grad for t in self._kept), "moments and masters take no gradients", 1)
        self._count = torch.tensor([int(step)], dtype=torch.int32, device=first.device) if capturable else None
        self._steps = int(step)

    def _lay_out(self):
        """The library's arrays of the tensors' addresses: the weights as they are now (a program
        may have put others into the list), moments and masters"""
        for what, tensors, dtype in self._state:
            self._listed(tensors, dtype, what)
        written = self.params + self._kept
        held = [t.detach() for t in written]
        spans = sorted((t.data_ptr(), t.numel() * t.element_size()) for t in written if t.numel())
        for (at, size), (nxt, _) in zip(spans, spans[1:]):
            _need(at + size <= nxt, "weights, moments and masters must not overlap", 1)
        self._seen, self._written, self._held = list(self.params), written, held   # (the addresses stay valid)
        self._arrays = [array("Q", map(_pointer, tensors)) for _, tensors, _ in self._state]
        self._at = [a.buffer_info()[0] for a in self._arrays] + [None] * (4 - len(self._arrays))

    def _new(self, make):
        """fp32 tensors of the weights' shapes in one buffer, each at 256 bytes"""
        sizes = [(p.numel() + 63) // 64 * 64 for p in self.params]
        flat = make(sum(sizes), dtype=torch.float32, device=self.params[0].device)
        return [b[:p.numel()].view(p.shape) for b, p in zip(flat.split(sizes), self.params)]

    def _listed(self, tensors, dtype, what: str):
        _need(len(tensors) == len(self._shapes), f"{what}: {len(self._shapes)} tensors expected, {len(tensors)} given")
        for i, (t, shape) in enumerate(zip(tensors, self._shapes)):
            if not isinstance(t, torch.Tensor):
                raise T2IError(1, f"{what}: entry {i} is no tensor, but {type(t).__name__}")
            if t.get_device() != self._dev:
                raise T2IError(1, f"{what}: tensors must be on the first weight's device")
            if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
                raise T2IError(2, f"{what}: expected {tuple(shape)} {dtype}, contiguous, got {tuple(t.shape)} {t.dtype}")

    @property
    def steps(self) -> int:
        """Steps taken so far (with ``capturable`` read from the device)"""
        return self._steps if self._count is None else int(self._count)

    def step(self, grads: Sequence[torch.Tensor], *, lr: Union[float, torch.Tensor, None] = None,
             grad_scale: Optional[torch.Tensor] = None, stream=None) -> None:
        """One step with the gradients of all weights, of one type (bf16 or fp32) and the weights'
        shapes (a weight that took no part has a gradient of zeros, not None).  ``lr``: instead of
        the constructor's, a number or one fp32 value on the device; ``grad_scale``: one fp32 value
        on the device that the gradients are multiplied by (the factor of a clipped norm).  Refused
        while gradients of a weight are recorded, like any operation in place on a leaf: call it
        under ``torch.no_grad()``."""
        dev = self._dev
        if _elsewhere(dev, stream):
            with _switch(dev, stream):
                return self.step(grads, lr=lr, grad_scale=grad_scale)
        if not isinstance(grads, (list, tuple)):
            _need(isinstance(grads, Iterable) and not isinstance(grads, torch.Tensor), "gradients must be a sequence", 1)
            grads = list(grads)
        first = grads[0] if len(grads) else None
        kind = _DTYPES.get(first.dtype) if isinstance(first, torch.Tensor) else None
        _need(kind is not None, "gradients of all weights, bf16 or fp32", 1)
        # (as lists and sets: the checks of a hundred tensors one by one take longer than the step)
        try:
            fit = (list(map(_shape, grads)) == self._shapes and set(map(_device_of, grads)) == {dev}
                   and set(map(_dtype, grads)) == {first.dtype} and all(map(_whole, grads)))
        except (AttributeError, TypeError):   # (no tensor)
            fit = False
        if not fit:
            self._listed(grads, first.dtype, "grads")
        try:
            at_rest = (len(self.params) == len(self._seen) and all(map(is_, self.params, self._seen))
                       and array("Q", map(_pointer, self.params)) == self._arrays[0])
        except TypeError:
            at_rest = False
        if not at_rest:
            self._lay_out()
        if torch.is_grad_enabled():
            _need(True not in map(_requires_grad, self.params) and True not in map(_requires_grad, grads),
                  "a tensor requires a gradient, which this call does not record: call under torch.no_grad()", 1)
        if getattr(forward_ad, "_current_level", 0) >= 0:   # (within a dual level)
            _need(all(forward_ad.unpack_dual(t).tangent is None for t in (*self._written, *grads)),
                  "a tensor carries a tangent, which this call does not pass on", 1)
        on_device = isinstance(lr, torch.Tensor)
        lr_at = _scalar(lr if on_device else None, dev, "lr")
        scale_at = _scalar(grad_scale, dev, "grad_scale")
        rate = 0.0 if on_device else float(self.lr if lr is None else lr)
        _need(math.isfinite(rate), "lr must be finite", 1)
        count = None
        if self._count is not None:
            with torch.no_grad():
                self._count += 1
            count = self._count.data_ptr()
        else:
            _need(not torch.cuda.is_current_stream_capturing(),
                  "a captured step needs capturable=True: its count would stand still in the graph", 1)
        p, m, v, masters = self._at
        at = array("Q", map(_pointer, grads))
        try:
            _check(load().t2i_op_adamw_step(
                self._type, kind, len(self.params), self._numel, p, at.buffer_info()[0], m, v, masters, rate,
                self.betas[0], self.betas[1], self.eps, self.weight_decay, self._steps + 1, lr_at, count, scale_at,
                _stream(dev)))
        except T2IError:
            if self._count is not None:   # (no step was taken)
                self._count -= 1
            raise
        self._steps += 1
        torch.autograd.graph.increment_version(self._written)
