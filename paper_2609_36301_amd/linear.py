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
from .layer import _call, _check, _device, _ptr, _size, _workspace

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
    _lib.check(_lib.load().more_expert_linear_plan(T, K, N, M, k, _KINDS[kind], ctypes.byref(plan)),
               "more_expert_linear_plan")
    return {name: getattr(plan, name) for name, _ in plan._fields_}


def _spec(T, K, N, M, k, dtype=torch.bfloat16):
    i32, f32 = torch.int32, torch.float32
    return {"x": (dtype, (T, K)), "q": (dtype, (T, K)), "Wt": (dtype, (M, N, K)), "Wq": (dtype, (M, N, K)),
            "idx": (i32, (T, k)), "offsets": (i32, (M + 1,)), "sorted": (i32, (T * k,)),
            "dy": (torch.bfloat16, (T * k, N)), "q_scale": (f32, (T,)), "w_scale": (f32, (M, N)), "gate": (f32, (T, k))}


def _shape(x, Wt, idx, names=("x", "Wt", "idx")):
    for name, t, dim in zip(names, (x, Wt, idx), (2, 3, 2)):
        if not isinstance(t, torch.Tensor):
            raise TypeError("%s must be a torch.Tensor" % name)
        if t.dim() != dim:
            raise ValueError("%s must have %d dimensions, got %s" % (name, dim, tuple(t.shape)))
    return x.shape[0], x.shape[1], Wt.shape[1], Wt.shape[0], idx.shape[1]


class _Checked:
    """The shape of a call, and the check of its tensors against it."""

    def _checks(self, **tensors):
        for name, t in tensors.items():
            dtype, shape = self.spec[name]
            _check(name, t, dtype, shape, self.device)


class ExpertLinear(_Checked):
    """Pre-allocated output and workspace for repeated expert_linear calls with one shape."""

    def __init__(self, T: int, K: int, N: int, M: int, k: int, *, out_dtype=torch.bfloat16, device=None):
        self.shape, self.spec, self.y_bits = (T, K, N, M, k), _spec(T, K, N, M, k), _y_bits(out_dtype)
        self.device = _device(device)
        self.workspace_bytes = expert_linear_workspace_size(*self.shape)
        self.workspace = _workspace(self.workspace_bytes, self.device)
        self.y = torch.empty((T * k, N), dtype=out_dtype, device=self.device)

    def __call__(self, x, Wt, idx, offsets, sorted) -> torch.Tensor:
        self._checks(x=x, Wt=Wt, idx=idx, offsets=offsets, sorted=sorted)
        _call("more_expert_linear", self.device, _ptr(x), _ptr(Wt), *self.shape, _ptr(idx), _ptr(offsets),
              _ptr(sorted), _ptr(self.y), self.y_bits, _ptr(self.workspace), self.workspace_bytes)
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


class ExpertLinearBackward(_Checked):
    """Pre-allocated gradients and workspace for repeated expert_linear_backward calls with one shape; either
    gradient may be left out."""

    def __init__(self, T: int, K: int, N: int, M: int, k: int, *, need_dx: bool = True, need_dW: bool = True, device=None):
        if not (need_dx or need_dW):
            raise ValueError("need_dx or need_dW must be set")
        self.shape, self.spec = (T, K, N, M, k), _spec(T, K, N, M, k)
        self.device = dev = _device(device)
        self.workspace_bytes = expert_linear_backward_workspace_size(*self.shape)
        self.workspace = _workspace(self.workspace_bytes, dev)
        self.dx = torch.empty((T, K), dtype=torch.bfloat16, device=dev) if need_dx else None
        self.dWt = torch.empty((M, N, K), dtype=torch.bfloat16, device=dev) if need_dW else None

    def __call__(self, x, Wt, idx, offsets, sorted, dy) -> LinearGradients:
        self._checks(x=x, Wt=Wt, idx=idx, offsets=offsets, sorted=sorted, dy=dy)
        _call("more_expert_linear_backward", self.device, _ptr(x), _ptr(Wt), *self.shape, _ptr(idx), _ptr(offsets),
              _ptr(sorted), _ptr(dy), _ptr(self.dx), _ptr(self.dWt), _ptr(self.workspace), self.workspace_bytes)
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


class QuantizeRows:
    """Pre-allocated outputs for repeated quantize_rows calls with one shape (T rows of `width` values; gated: of
    2 width)."""

    def __init__(self, T: int, width: int, *, gated: bool = False, device=None):
        self.shape, self.gated, self.device = (T, width), bool(gated), _device(device)
        self.q = torch.empty((T, width), dtype=torch.int8, device=self.device)
        self.scale = torch.empty((T,), dtype=torch.float32, device=self.device)

    def __call__(self, x) -> QuantizedRows:
        T, width = self.shape
        _check("x", x, torch.bfloat16, (T, 2 * width if self.gated else width), self.device)
        _call("more_quantize_rows", self.device, _ptr(x), T, width, int(self.gated), _ptr(self.q), _ptr(self.scale))
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


class ExpertLinearQ8(_Checked):
    """Pre-allocated output and workspace for repeated expert_linear_q8 calls with one shape."""

    def __init__(self, T: int, K: int, N: int, M: int, k: int, *, out_dtype=torch.bfloat16, device=None):
        self.shape, self.spec, self.y_bits = (T, K, N, M, k), _spec(T, K, N, M, k, torch.int8), _y_bits(out_dtype)
        self.device = _device(device)
        self.workspace_bytes = expert_linear_q8_workspace_size(*self.shape)
        self.workspace = _workspace(self.workspace_bytes, self.device)
        self.y = torch.empty((T * k, N), dtype=out_dtype, device=self.device)

    def __call__(self, q, q_scale, Wq, w_scale, idx, offsets, sorted, gate=None) -> torch.Tensor:
        self._checks(q=q, q_scale=q_scale, Wq=Wq, w_scale=w_scale, idx=idx, offsets=offsets, sorted=sorted)
        if gate is not None:
            self._checks(gate=gate)
        _call("more_expert_linear_q8", self.device, _ptr(q), _ptr(q_scale), _ptr(Wq), _ptr(w_scale), *self.shape,
              _ptr(idx), _ptr(offsets), _ptr(sorted), _ptr(gate), _ptr(self.y), self.y_bits, _ptr(self.workspace),
              self.workspace_bytes)
        return self.y


def expert_linear_q8(q, q_scale, Wq, w_scale, idx, offsets, sorted, gate=None, *, out_dtype=torch.bfloat16) -> torch.Tensor:
    """expert_linear of rows and weights in 8-bit integers: q [T][K] and Wq [M][N][K] int8 with their scales [T] and
    [M][N], times gate [T][k] where it is given (more_expert_linear_q8)."""
    call = ExpertLinearQ8(*_shape(q, Wq, idx, ("q", "Wq", "idx")), out_dtype=out_dtype, device=q.device)
    return call(q, q_scale, Wq, w_scale, idx, offsets, sorted, gate)
