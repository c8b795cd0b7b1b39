"""Python binding of the distillation from a teacher's top logits (see include/more.h for the formulas and limits).

A low-rank router learns from a full-rank one: the teacher's entries are the latter's selection, the student's
logits over all experts two linear maps (M = 1):

    teacher = route_fullrank(x, Wt, k, topval=True)
    d = distill_loss(logits, teacher.idx, teacher.topval, temperature=2.0)       # d.loss [T]
    dlogits = distill_backward(logits, d.m, d.Z, teacher.idx, teacher.topval, dloss, temperature=2.0)

or both at once, where the gradient of each loss is known beforehand:

    d = distill_loss(logits, teacher.idx, teacher.topval, weight, temperature=2.0, gradient=True)   # d.loss, d.dlogits

As in `layer`, every function only checks tensor metadata, allocates outputs with torch on the tensors' device, and
passes raw device pointers and that device's current HIP stream to libmore.so; nothing is recorded for torch's
autograd.  The classes hold outputs for repeated calls with one shape: a call only launches, can be captured in a
HIP graph, and overwrites the outputs of the call before; calls of one object must be ordered on one stream.
"""
from __future__ import annotations

import dataclasses
from typing import Optional

import torch

from .layer import _call, _check, _device, _ptr

_BITS = {torch.bfloat16: 16, torch.float32: 32}


@dataclasses.dataclass
class Distillation:
    loss: torch.Tensor               # float32 [T]
    m: torch.Tensor                  # float32 [T], the largest logit
    Z: torch.Tensor                  # float32 [T], sum of exp((z - m) / temperature)
    dlogits: Optional[torch.Tensor]  # the logits' type, [T][V]


class _Rows:
    """Rows of V logits, ld apart, and their teacher's entries."""

    def __init__(self, T: int, V: int, k: int, dtype, temperature: float, ld, inplace: bool, gradient: bool, device):
        if dtype not in _BITS:
            raise TypeError("logits must be float32 or bfloat16, got %s" % dtype)
        self.shape, self.dtype, self.bits = (T, V, k), dtype, _BITS[dtype]
        self.ld = V if ld is None else int(ld)
        if self.ld < V:
            raise ValueError("ld must be at least V = %d, got %d" % (V, self.ld))
        self.temperature, self.inplace, self.gradient = float(temperature), bool(inplace), bool(gradient)
        self.device = _device(device)
        self.dlogits = None
        if gradient and not inplace:
            self.dlogits = torch.empty((T, self.ld), dtype=dtype, device=self.device)[:, :V]

    def _check_rows(self, logits, teacher_idx, teacher_val):
        T, V, k = self.shape
        if not isinstance(logits, torch.Tensor):
            raise TypeError("logits must be a torch.Tensor")
        if logits.dtype != self.dtype:
            raise TypeError("logits must be %s, got %s" % (self.dtype, logits.dtype))
        if logits.shape != (T, V) or (V > 1 and logits.stride(1) != 1) or (T > 1 and logits.stride(0) != self.ld):
            raise ValueError("logits must be %d rows of %d values, %d apart, got %s with strides %s"
                             % (T, V, self.ld, tuple(logits.shape), tuple(logits.stride())))
        if logits.device != self.device:
            raise ValueError("logits must be on %s, got %s" % (self.device, logits.device))
        _check("teacher_idx", teacher_idx, torch.int32, (T, k), self.device)
        _check("teacher_val", teacher_val, torch.float32, (T, k), self.device)

    def _out(self, logits):
        return None if not self.gradient else logits if self.inplace else self.dlogits


class Distill(_Rows):
    """Pre-allocated outputs for repeated distill_loss calls with one shape: T rows of V logits that lie `ld` apart
    (V by default), k teacher entries each.  gradient: the weighted gradient comes with the loss; inplace: over the
    logits."""

    def __init__(self, T: int, V: int, k: int, *, dtype=torch.bfloat16, temperature: float = 1.0, ld: Optional[int] = None,
                 gradient: bool = False, inplace: bool = False, device=None):
        super().__init__(T, V, k, dtype, temperature, ld, inplace, gradient, device)
        self.loss, self.m, self.Z = (torch.empty((T,), dtype=torch.float32, device=self.device) for _ in range(3))

    def __call__(self, logits, teacher_idx, teacher_val, weight=None) -> Distillation:
        self._check_rows(logits, teacher_idx, teacher_val)
        T, V, k = self.shape
        if weight is not None:
            if not self.gradient:
                raise ValueError("weight is of use only where the gradient is asked for")
            _check("weight", weight, torch.float32, (T,), self.device)
        out = self._out(logits)
        _call("more_distill", self.device, _ptr(logits), self.bits, T, V, self.ld, _ptr(teacher_idx), _ptr(teacher_val), k,
              self.temperature, _ptr(weight), _ptr(self.loss), _ptr(self.m), _ptr(self.Z), _ptr(out), self.ld)
        return Distillation(self.loss, self.m, self.Z, out)


class DistillBackward(_Rows):
    """Pre-allocated gradient for repeated distill_backward calls with one shape (as for Distill)."""

    def __init__(self, T: int, V: int, k: int, *, dtype=torch.bfloat16, temperature: float = 1.0, ld: Optional[int] = None,
                 inplace: bool = False, device=None):
        super().__init__(T, V, k, dtype, temperature, ld, inplace, True, device)

    def __call__(self, logits, m, Z, teacher_idx, teacher_val, dloss) -> torch.Tensor:
        self._check_rows(logits, teacher_idx, teacher_val)
        T, V, k = self.shape
        for name, t in (("m", m), ("Z", Z), ("dloss", dloss)):
            _check(name, t, torch.float32, (T,), self.device)
        out = self._out(logits)
        _call("more_distill_backward", self.device, _ptr(logits), self.bits, T, V, self.ld, _ptr(m), _ptr(Z),
              _ptr(teacher_idx), _ptr(teacher_val), k, self.temperature, _ptr(dloss), _ptr(out), self.ld)
        return out


def _rows_of(logits, teacher_idx):
    for name, t in (("logits", logits), ("teacher_idx", teacher_idx)):
        if not isinstance(t, torch.Tensor) or t.dim() != 2:
            raise ValueError("%s must be a 2-D tensor" % name)
    T, V = logits.shape
    ld = logits.stride(0) if T > 1 else V
    if ld < V:
        raise ValueError("rows of logits must not overlap, got strides %s" % (tuple(logits.stride()),))
    return (T, V, teacher_idx.shape[1]), {"dtype": logits.dtype, "ld": ld, "device": logits.device}


def distill_loss(logits, teacher_idx, teacher_val, weight=None, *, temperature: float = 1.0, gradient: bool = False) -> Distillation:
    """Per row t of the logits [T][V] (float32 or bfloat16, rows may lie apart): temperature^2 times the divergence of
    softmax(logits / temperature) from softmax(teacher_val / temperature) over the classes teacher_idx [T][k] int32;
    entries with an id outside [0, V) are left out.  gradient: with the gradient of sum(weight * loss) (more_distill)."""
    shape, options = _rows_of(logits, teacher_idx)
    call = Distill(*shape, temperature=temperature, gradient=gradient, **options)
    return call(logits, teacher_idx, teacher_val, weight)


def distill_backward(logits, m, Z, teacher_idx, teacher_val, dloss, *, temperature: float = 1.0) -> torch.Tensor:
    """The gradient of distill_loss with respect to the logits, given its m and Z and the gradient with respect to each
    loss (more_distill_backward)."""
    shape, options = _rows_of(logits, teacher_idx)
    call = DistillBackward(*shape, temperature=temperature, **options)
    return call(logits, m, Z, teacher_idx, teacher_val, dloss)
