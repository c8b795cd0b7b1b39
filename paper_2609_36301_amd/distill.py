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

import ctypes
import dataclasses
from typing import Optional

import torch

from . import _lib
from .layer import _ptr
from .linear import _Call

_BITS = {torch.bfloat16: 16, torch.float32: 32}


@dataclasses.dataclass
class Distillation:
    loss: torch.Tensor               # float32 [T]
    m: torch.Tensor                  # float32 [T], the largest logit
    Z: torch.Tensor                  # float32 [T], sum of exp((z - m) / temperature)
    dlogits: Optional[torch.Tensor]  # the logits' type, [T][V]


class _Rows(_Call):
    """Rows of V logits, ld apart, and their teacher's entries."""

    _function, _vectors = "", ()

    def __init__(self, T: int, V: int, k: int, dtype, temperature: float, ld, inplace: bool, gradient: bool, device):
        if dtype not in _BITS:
            raise TypeError("logits must be float32 or bfloat16, got %s" % dtype)
        self.shape, self.dtype, self.bits = (T, V, k), dtype, _BITS[dtype]
        self.ld = V if ld is None else int(ld)
        if self.ld < V:
            raise ValueError("ld must be at least V = %d, got %d" % (V, self.ld))
        self.temperature, self.inplace, self.gradient = float(temperature), bool(inplace), bool(gradient)
        f32, i64 = torch.float32, ctypes.c_int64
        self._rows = (ctypes.c_int32(self.bits), _lib.integer(T, self._function, i64), _lib.integer(V, self._function),
                      _lib.integer(self.ld, self._function, i64))
        self._entries = (_lib.integer(k, self._function), ctypes.c_float(self.temperature))
        self._prepare(self._function, device, teacher_idx=(torch.int32, (T, k)), teacher_val=(f32, (T, k)),
                      **{name: (f32, (T,)) for name in self._vectors})
        self._strides = (self.ld if T > 1 else None, 1 if V > 1 else None)
        self.dlogits = None
        if gradient and not inplace:
            self.dlogits = torch.empty((T, self.ld), dtype=dtype, device=self.device)[:, :V]

    def _check_rows(self, logits):
        T, V, k = self.shape
        if not isinstance(logits, torch.Tensor):
            raise TypeError("logits must be a torch.Tensor")
        if logits.dtype is not self.dtype:
            raise TypeError("logits must be %s, got %s" % (self.dtype, logits.dtype))
        strides = logits.stride()
        if logits.shape != (T, V) or strides[0] != (self._strides[0] or strides[0]) or strides[1] != (self._strides[1] or strides[1]):
            raise ValueError("logits must be %d rows of %d values, %d apart, got %s with strides %s"
                             % (T, V, self.ld, tuple(logits.shape), tuple(strides)))
        if logits.get_device() != self.device.index:
            raise ValueError("logits must be on %s, got %s" % (self.device, logits.device))

    def _out(self, logits):
        return None if not self.gradient else logits if self.inplace else self.dlogits


class Distill(_Rows):
    """Pre-allocated outputs for repeated distill_loss calls with one shape: T rows of V logits that lie `ld` apart
    (V by default), k teacher entries each.  gradient: the weighted gradient comes with the loss; inplace: over the
    logits."""

    _function, _vectors = "more_distill", ("weight",)

    def __init__(self, T: int, V: int, k: int, *, dtype=torch.bfloat16, temperature: float = 1.0, ld: Optional[int] = None,
                 gradient: bool = False, inplace: bool = False, device=None):
        super().__init__(T, V, k, dtype, temperature, ld, inplace, gradient, device)
        self.loss, self.m, self.Z = (torch.empty((T,), dtype=torch.float32, device=self.device) for _ in range(3))

    def __call__(self, logits, teacher_idx, teacher_val, weight=None) -> Distillation:
        self._check_rows(logits)
        if weight is None:
            self._check_tensors(teacher_idx, teacher_val)
        elif not self.gradient:
            raise ValueError("weight is of use only where the gradient is asked for")
        else:
            self._check_tensors(teacher_idx, teacher_val, weight)
        out = self._out(logits)
        self._launch(logits.data_ptr(), *self._rows, teacher_idx.data_ptr(), teacher_val.data_ptr(), *self._entries,
                     _ptr(weight), self.loss.data_ptr(), self.m.data_ptr(), self.Z.data_ptr(), _ptr(out), self.ld)
        return Distillation(self.loss, self.m, self.Z, out)


class DistillBackward(_Rows):
    """Pre-allocated gradient for repeated distill_backward calls with one shape (as for Distill)."""

    _function, _vectors = "more_distill_backward", ("m", "Z", "dloss")

    def __init__(self, T: int, V: int, k: int, *, dtype=torch.bfloat16, temperature: float = 1.0, ld: Optional[int] = None,
                 inplace: bool = False, device=None):
        super().__init__(T, V, k, dtype, temperature, ld, inplace, True, device)

    def __call__(self, logits, m, Z, teacher_idx, teacher_val, dloss) -> torch.Tensor:
        self._check_rows(logits)
        self._check_tensors(teacher_idx, teacher_val, m, Z, dloss)
        out = self._out(logits)
        self._launch(logits.data_ptr(), *self._rows, m.data_ptr(), Z.data_ptr(), teacher_idx.data_ptr(),
                     teacher_val.data_ptr(), *self._entries, dloss.data_ptr(), out.data_ptr(), self.ld)
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
