"""Python binding of the experts' linear maps, in bf16 with their backward pass and in 8-bit integers (see
include/more.h for the formulas and limits).

    offsets, srt = dispatch_sort(sel.idx, M)
    y = expert_linear(x, Wt, sel.idx, offsets, srt)                       # [T k][N], a row per entry
    g = expert_linear_backward(x, Wt, sel.idx, offsets, srt, dy)          # g.dx, g.dWt

A map that follows takes the entries' rows as tokens with one entry each, and the same offsets and sorted; an
experts' block in 8-bit integers, as a program serves it:

    entries = sel.idx.view(-1, 1)
    W1q, W2q = quantize_rows(W1t), quantize_rows(W2t)                     # once: a scale per output channel
    xq = quantize_rows(xn)
    gu = expert_linear_q8(xq.q, xq.scale, W1q.q, W1q.scale, sel.idx, offsets, srt)           # [T k][2s]
    aq = quantize_rows(gu, gated=True)                                    # silu(g) u, in 8 bits
    y = expert_linear_q8(aq.q, aq.scale, W2q.q, W2q.scale, entries, offsets, srt, sel.gate.view(-1, 1))

As in `layer`, every function only checks tensor metadata, allocates outputs and workspace with torch on the
tensors' device, and passes raw device pointers and that device's current HIP stream to libmore.so; nothing is
recorded for torch's autograd.  The classes hold outputs and workspace for repeated calls with one shape: a call
only launches, can be captured in a HIP graph, and overwrites the outputs of the call before; calls of one object
must be ordered on one stream.
"""
from __future__ import annotations

import ctypes
import dataclasses
from typing import Optional

import torch

from . import _lib
from .layer import _check, _device, _ptr, _size, _stream, _workspace

_Y_BITS = {torch.bfloat16: 16, torch.float32: 32}
_KINDS = {"linear": 0, "backward": 1, "q8": 2}


def _y_bits(dtype) -> int:
    if dtype not in _Y_BITS:
        raise TypeError("the output must be bfloat16 or float32, got %s" % dtype)
    return _Y_BITS[dtype]


def expert_linear_workspace_size(T: int, K: int, N: int, M: int, k: int) -> int:
    return _size("more_expert_linear_workspace_size", T, K, N, M, k)


def expert_linear_backward_workspace_size(T: int, K: int, N: int, M: int, k: int) -> int:
    return _size("more_expert_linear_backward_workspace_size", T, K, N, M, k)


def expert_linear_q8_workspace_size(T: int, K: int, N: int, M: int, k: int) -> int:
    return _size("more_expert_linear_q8_workspace_size", T, K, N, M, k)


def expert_linear_plan(T: int, K: int, N: int, M: int, k: int, kind: str = "linear") -> dict[str, int]:
    """The form in which a map ("linear", "backward" or "q8") runs this shape: the fields of more_linear_plan."""
    plan = _lib.LinearPlan()
    _lib.query("more_expert_linear_plan", T, K, N, M, k, _KINDS[kind], ctypes.byref(plan))
    return {name: getattr(plan, name) for name, _ in plan._fields_}


def _shape(x, Wt, idx, names=("x", "Wt", "idx")):
    for name, t, dim in zip(names, (x, Wt, idx), (2, 3, 2)):
        if not isinstance(t, torch.Tensor):
            raise TypeError("%s must be a torch.Tensor" % name)
        if t.dim() != dim:
            raise ValueError("%s must have %d dimensions, got %s" % (name, dim, tuple(t.shape)))
    return x.shape[0], x.shape[1], Wt.shape[1], Wt.shape[0], idx.shape[1]


_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


class _Call:
    """A library call of one shape: what its tensors have to be, and the arguments that stay.  (The host takes longer than a
    single token's kernel, most of it for checking tensors: 4.1 us for five one attribute at a time, 2.5 so.)"""

    def _prepare(self, name: str, device, **tensors):
        """tensors: dtype and shape by name, in the call's order."""
        self.device = _device(device)
        self._name, self._fn = name, getattr(_lib.load(), name)
        self._names = list(tensors)
        self._spec = [(dtype, torch.Size(shape)) for dtype, shape in tensors.values()]

    def _check_tensors(self, *tensors):
        index = self.device.index
        try:
            for (dtype, shape), t in zip(self._spec, tensors):
                if not (t.dtype is dtype and t.shape == shape and t.get_device() == index and t.is_contiguous()):
                    break
            else:
                return
        except AttributeError:
            pass  # (no tensor)
        for name, (dtype, shape), t in zip(self._names, self._spec, tensors):
            _check(name, t, dtype, shape, self.device)

    def _launch(self, *args):
        """The call on the device's current stream (the library works on the current device)."""
        index = self.device.index
        stream = _stream(index)
        if _current_device() == index:
            status = self._fn(*args, stream)
        else:
            with torch.cuda.device(self.device):
                status = self._fn(*args, stream)
        if status:
            _lib.check(status, self._name)


def _sizes(name, T, *sizes):
    return (_lib.integer(T, name, ctypes.c_int64),) + tuple(_lib.integer(size, name) for size in sizes)


def _selection(T, M, k):
    i32 = torch.int32
    return {"idx": (i32, (T, k)), "offsets": (i32, (M + 1,)), "sorted": (i32, (T * k,))}


class ExpertLinear(_Call):
    """Pre-allocated output and workspace for repeated expert_linear calls with one shape."""

    def __init__(self, T: int, K: int, N: int, M: int, k: int, *, out_dtype=torch.bfloat16, device=None):
        bf16 = torch.bfloat16
        self.shape, self.y_bits = (T, K, N, M, k), _y_bits(out_dtype)
        self._sizes = _sizes("more_expert_linear", T, K, N, M, k)
        self._prepare("more_expert_linear", device, x=(bf16, (T, K)), Wt=(bf16, (M, N, K)), **_selection(T, M, k))
        self.workspace_bytes = expert_linear_workspace_size(*self.shape)
        self.workspace = _workspace(self.workspace_bytes, self.device)
        self.y = torch.empty((T * k, N), dtype=out_dtype, device=self.device)

    def __call__(self, x, Wt, idx, offsets, sorted) -> torch.Tensor:
        self._check_tensors(x, Wt, idx, offsets, sorted)
        self._launch(x.data_ptr(), Wt.data_ptr(), *self._sizes, idx.data_ptr(), offsets.data_ptr(), sorted.data_ptr(),
                     self.y.data_ptr(), self.y_bits, self.workspace.data_ptr(), self.workspace_bytes)
        return self.y


def expert_linear(x, Wt, idx, offsets, sorted, *, out_dtype=torch.bfloat16) -> torch.Tensor:
    """y [T k][N]: row t k + j is x[t] Wt[idx[t][j]]^T; zero rows for ids outside [0, M).  offsets and sorted are
    dispatch_sort(idx, M)'s (more_expert_linear)."""
    call = ExpertLinear(*_shape(x, Wt, idx), out_dtype=out_dtype, device=x.device)
    return call(x, Wt, idx, offsets, sorted)


@dataclasses.dataclass
class LinearGradients:
    """Gradients of expert_linear."""
    dx: Optional[torch.Tensor]   # bfloat16 [T][K]
    dWt: Optional[torch.Tensor]  # bfloat16 [M][N][K]


class ExpertLinearBackward(_Call):
    """Pre-allocated gradients and workspace for repeated expert_linear_backward calls with one shape; either
    gradient may be left out."""

    def __init__(self, T: int, K: int, N: int, M: int, k: int, *, need_dx: bool = True, need_dW: bool = True, device=None):
        if not (need_dx or need_dW):
            raise ValueError("need_dx or need_dW must be set")
        bf16 = torch.bfloat16
        self.shape, self._sizes = (T, K, N, M, k), _sizes("more_expert_linear_backward", T, K, N, M, k)
        self._prepare("more_expert_linear_backward", device, x=(bf16, (T, K)), Wt=(bf16, (M, N, K)), **_selection(T, M, k),
                      dy=(bf16, (T * k, N)))
        dev = self.device
        self.workspace_bytes = expert_linear_backward_workspace_size(*self.shape)
        self.workspace = _workspace(self.workspace_bytes, dev)
        self.dx = torch.empty((T, K), dtype=bf16, device=dev) if need_dx else None
        self.dWt = torch.empty((M, N, K), dtype=bf16, device=dev) if need_dW else None

    def __call__(self, x, Wt, idx, offsets, sorted, dy) -> LinearGradients:
        self._check_tensors(x, Wt, idx, offsets, sorted, dy)
        self._launch(x.data_ptr(), Wt.data_ptr(), *self._sizes, idx.data_ptr(), offsets.data_ptr(), sorted.data_ptr(),
                     dy.data_ptr(), _ptr(self.dx), _ptr(self.dWt), self.workspace.data_ptr(), self.workspace_bytes)
        return LinearGradients(self.dx, self.dWt)


def expert_linear_backward(x, Wt, idx, offsets, sorted, dy, *, need_dx: bool = True, need_dW: bool = True) -> LinearGradients:
    """Gradients of expert_linear given dy [T k][N] bf16, the gradient with respect to y
    (more_expert_linear_backward)."""
    call = ExpertLinearBackward(*_shape(x, Wt, idx), need_dx=need_dx, need_dW=need_dW, device=x.device)
    return call(x, Wt, idx, offsets, sorted, dy)


# ---------------------------------------------------------------------------------- 8-bit integers
@dataclasses.dataclass
class QuantizedRows:
    """x is about q times its row's scale."""
    q: torch.Tensor      # int8, x's shape (gated: half its last dimension)
    scale: torch.Tensor  # float32, x's shape without the last dimension


class QuantizeRows(_Call):
    """Pre-allocated outputs for repeated quantize_rows calls with one shape (T rows of `width` values; gated: of
    2 width)."""

    def __init__(self, T: int, width: int, *, gated: bool = False, device=None):
        self.shape, self.gated = (T, width), bool(gated)
        self._sizes = _sizes("more_quantize_rows", T, width, self.gated)
        self._prepare("more_quantize_rows", device, x=(torch.bfloat16, (T, 2 * width if gated else width)))
        self.q = torch.empty((T, width), dtype=torch.int8, device=self.device)
        self.scale = torch.empty((T,), dtype=torch.float32, device=self.device)

    def __call__(self, x) -> QuantizedRows:
        self._check_tensors(x)
        self._launch(x.data_ptr(), *self._sizes, self.q.data_ptr(), self.scale.data_ptr())
        return QuantizedRows(self.q, self.scale)


def quantize_rows(x, *, gated: bool = False) -> QuantizedRows:
    """The rows (last dimension) of x, bf16 with any leading dimensions, in 8-bit integers with a scale each; gated:
    a row is [g u] and silu(g) u is quantised (more_quantize_rows)."""
    if not isinstance(x, torch.Tensor):
        raise TypeError("x must be a torch.Tensor")
    if x.dim() < 1 or x.shape[-1] == 0 or not x.is_contiguous():
        raise ValueError("x must be a contiguous tensor of rows, got %s" % (tuple(x.shape),))
    if gated and x.shape[-1] % 2:
        raise ValueError("gated rows have an even number of values, got %d" % x.shape[-1])
    lead, width = x.shape[:-1], x.shape[-1] // 2 if gated else x.shape[-1]
    rows = x.view(-1, x.shape[-1])
    out = QuantizeRows(rows.shape[0], width, gated=gated, device=x.device)(rows)
    return QuantizedRows(out.q.view(*lead, width), out.scale.view(lead))


class ExpertLinearQ8(_Call):
    """Pre-allocated output and workspace for repeated expert_linear_q8 calls with one shape."""

    def __init__(self, T: int, K: int, N: int, M: int, k: int, *, out_dtype=torch.bfloat16, device=None):
        i8, f32 = torch.int8, torch.float32
        self.shape, self.y_bits = (T, K, N, M, k), _y_bits(out_dtype)
        self._sizes = _sizes("more_expert_linear_q8", T, K, N, M, k)
        self._prepare("more_expert_linear_q8", device, q=(i8, (T, K)), q_scale=(f32, (T,)), Wq=(i8, (M, N, K)),
                      w_scale=(f32, (M, N)), **_selection(T, M, k), gate=(f32, (T, k)))
        self.workspace_bytes = expert_linear_q8_workspace_size(*self.shape)
        self.workspace = _workspace(self.workspace_bytes, self.device)
        self.y = torch.empty((T * k, N), dtype=out_dtype, device=self.device)

    def __call__(self, q, q_scale, Wq, w_scale, idx, offsets, sorted, gate=None) -> torch.Tensor:
        given = (q, q_scale, Wq, w_scale, idx, offsets, sorted)
        self._check_tensors(*given if gate is None else (*given, gate))
        self._launch(q.data_ptr(), q_scale.data_ptr(), Wq.data_ptr(), w_scale.data_ptr(), *self._sizes, idx.data_ptr(),
                     offsets.data_ptr(), sorted.data_ptr(), _ptr(gate), self.y.data_ptr(), self.y_bits,
                     self.workspace.data_ptr(), self.workspace_bytes)
        return self.y


def expert_linear_q8(q, q_scale, Wq, w_scale, idx, offsets, sorted, gate=None, *, out_dtype=torch.bfloat16) -> torch.Tensor:
    """expert_linear of rows and weights in 8-bit integers: q [T][K] and Wq [M][N][K] int8 with their scales [T] and
    [M][N], times gate [T][k] where it is given (more_expert_linear_q8)."""
    call = ExpertLinearQ8(*_shape(q, Wq, idx, ("q", "Wq", "idx")), out_dtype=out_dtype, device=q.device)
    return call(q, q_scale, Wq, w_scale, idx, offsets, sorted, gate)
