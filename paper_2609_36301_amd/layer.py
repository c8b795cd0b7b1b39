"""Python binding of the layer around the router: the experts' gated feed-forward block, the norms at
a block's ends and the clipping of gradients, each with its backward pass where it has one.

A layer as a program runs it (see include/more.h for the formulas and limits):

    xn = block_norm(r, w_before=w0).xn                    # norm before the first block
    sel = route_lowrank(xn, R1t, R2t, k)                  # the router
    offsets, srt = dispatch_sort(sel.idx, M)              # Sort + Count
    y = expert_ffn(xn, W1t, W2t, sel.idx, offsets, srt, sel.gate)
    end = block_norm(r, y, w_after=w1, w_before=w2)       # r' = alpha r + w1 u/rms(u), xn = w2 r'/rms(r')

As in `router`, every function only checks tensor metadata, allocates outputs and workspace with torch
on the tensors' device, and passes raw device pointers and that device's current HIP stream to
libmore.so.  The classes hold outputs and workspace for repeated calls with one shape: a call only
launches, can be captured in a HIP graph, and overwrites the outputs of the call before; calls of one
object must be ordered on one stream.

As the router's, these calls record nothing for torch's autograd, whatever requires_grad says: the
*_backward functions are the gradients, for a program to call or to wrap in a torch.autograd.Function.
"""
from __future__ import annotations

import ctypes
import dataclasses
from typing import Optional, Sequence

import torch

from . import _lib


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _device(device) -> torch.device:
    dev = torch.device(device or "cuda")
    if dev.type != "cuda":
        raise ValueError("device must be a GPU device, got %s" % dev)
    return dev if dev.index is not None else torch.device("cuda", torch.cuda.current_device())


def _good(t, dtype, shape, device) -> bool:
    return (isinstance(t, torch.Tensor) and t.dtype == dtype and t.shape == shape and t.device == device
            and t.is_contiguous())


def _check(name: str, t, dtype, shape, device):
    if _good(t, dtype, shape, device):
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.shape != shape or not t.is_contiguous():
        raise ValueError("%s must be a contiguous tensor of shape %s, got %s"
                         % (name, tuple(shape), tuple(t.shape)))
    raise ValueError("%s must be on %s, got %s" % (name, device, t.device))


# The handle of a device's current stream, by the device's index (without a Stream object around it, which
# takes 1.9 us, a quarter of a short call).
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _call(name: str, device: torch.device, *args):
    """The library call `name` on the device's current stream (the library works on the current device)."""
    stream = _stream(device.index)
    fn = getattr(_lib.load(), name)
    if torch.cuda.current_device() == device.index:
        st = fn(*args, stream)
    else:
        with torch.cuda.device(device):
            st = fn(*args, stream)
    _lib.check(st, name)


def _size(name: str, *args) -> int:
    n = ctypes.c_size_t(0)
    _lib.query(name, *args, ctypes.byref(n))
    return n.value


def _workspace(nbytes: int, device) -> torch.Tensor:
    return torch.empty((max(nbytes, 1),), dtype=torch.uint8, device=device)


# ---------------------------------------------------------------------------------- experts
# addends (of every call on the experts): 0 rounds the hidden units between the two products to one bf16 where there
# are many and to a sum of two where there are few; 2 takes two at every size (more_expert_ffn_ex).
def expert_ffn_workspace_size(T: int, h: int, s: int, M: int, k: int, addends: int = 0) -> int:
    return _size("more_expert_ffn_workspace_size_ex", T, h, s, M, k, addends)


def expert_ffn_backward_workspace_size(T: int, h: int, s: int, M: int, k: int, addends: int = 0) -> int:
    return _size("more_expert_ffn_backward_workspace_size_ex", T, h, s, M, k, addends)


def expert_ffn_plan(T: int, h: int, s: int, M: int, k: int, backward: bool = False, addends: int = 0) -> dict[str, int]:
    """The form in which expert_ffn (or its backward pass) runs this shape: the fields of more_expert_plan."""
    plan = _lib.ExpertPlan()
    _lib.query("more_expert_ffn_plan", T, h, s, M, k, addends, int(backward), ctypes.byref(plan))
    return {name: getattr(plan, name) for name, _ in plan._fields_}


def _ffn_spec(T, h, s, M, k):
    bf16, i32 = torch.bfloat16, torch.int32
    return (("x", bf16, (T, h)), ("W1t", bf16, (M, 2 * s, h)), ("W2t", bf16, (M, h, s)), ("idx", i32, (T, k)),
            ("offsets", i32, (M + 1,)), ("sorted", i32, (T * k,)), ("gate", torch.float32, (T, k)),
            ("du", bf16, (T, h)))


def _check_ffn(spec, device, *tensors):
    for (name, dtype, shape), t in zip(spec, tensors):
        if not (t is None and name == "gate"):
            _check(name, t, dtype, shape, device)


def _ffn_shape(x, W1t, W2t, idx):
    for name, t, dim in (("x", x, 2), ("W1t", W1t, 3), ("W2t", W2t, 3), ("idx", idx, 2)):
        if not isinstance(t, torch.Tensor):
            raise TypeError("%s must be a torch.Tensor" % name)
        if t.dim() != dim:
            raise ValueError("%s must have %d dimensions, got %s" % (name, dim, tuple(t.shape)))
    return x.shape[0], x.shape[1], W2t.shape[2], W1t.shape[0], idx.shape[1]


class ExpertFFN:
    """Pre-allocated output and workspace for repeated expert_ffn calls with one shape."""

    def __init__(self, T: int, h: int, s: int, M: int, k: int, *, addends: int = 0, device=None):
        self.shape, self.spec, self.addends = (T, h, s, M, k), _ffn_spec(T, h, s, M, k), addends
        self.device = _device(device)
        self.workspace_bytes = expert_ffn_workspace_size(*self.shape, addends)
        self.workspace = _workspace(self.workspace_bytes, self.device)
        self.y = torch.empty((T * k, h), dtype=torch.bfloat16, device=self.device)

    def __call__(self, x, W1t, W2t, idx, offsets, sorted, gate=None) -> torch.Tensor:
        _check_ffn(self.spec, self.device, x, W1t, W2t, idx, offsets, sorted, gate)
        _call("more_expert_ffn_ex", self.device, _ptr(x), _ptr(W1t), _ptr(W2t), *self.shape, self.addends,
              _ptr(idx), _ptr(offsets), _ptr(sorted), _ptr(gate), _ptr(self.y), _ptr(self.workspace),
              self.workspace_bytes)
        return self.y


def expert_ffn(x, W1t, W2t, idx, offsets, sorted, gate=None, *, addends: int = 0) -> torch.Tensor:
    """y [T k][h] bf16: row t k + j is gate[t][j] times the gated feed-forward block of expert
    idx[t][j] applied to x[t]; zero rows for ids outside [0, M).  offsets and sorted are
    dispatch_sort(idx, M)'s.  addends = 2 carries the hidden units as two bf16 addends at every size
    (more_expert_ffn_ex)."""
    shape = _ffn_shape(x, W1t, W2t, idx)
    return ExpertFFN(*shape, addends=addends, device=x.device)(x, W1t, W2t, idx, offsets, sorted, gate)


@dataclasses.dataclass
class ExpertGradients:
    """Gradients of expert_ffn."""
    dx: torch.Tensor               # bfloat16 [T][h]
    dW1t: torch.Tensor             # bfloat16 [M][2s][h]
    dW2t: torch.Tensor             # bfloat16 [M][h][s]
    dgate: Optional[torch.Tensor]  # float32 [T][k], None without gates


class ExpertFFNBackward:
    """Pre-allocated gradients and workspace for repeated expert_ffn_backward calls with one shape."""

    def __init__(self, T: int, h: int, s: int, M: int, k: int, *, addends: int = 0, device=None):
        self.shape, self.spec, self.addends = (T, h, s, M, k), _ffn_spec(T, h, s, M, k), addends
        self.device = dev = _device(device)
        self.workspace_bytes = expert_ffn_backward_workspace_size(*self.shape, addends)
        self.workspace = _workspace(self.workspace_bytes, dev)
        bf16 = torch.bfloat16
        self.dx = torch.empty((T, h), dtype=bf16, device=dev)
        self.dW1t = torch.empty((M, 2 * s, h), dtype=bf16, device=dev)
        self.dW2t = torch.empty((M, h, s), dtype=bf16, device=dev)
        self.dgate = torch.empty((T, k), dtype=torch.float32, device=dev)

    def __call__(self, x, W1t, W2t, idx, offsets, sorted, gate, du) -> ExpertGradients:
        _check_ffn(self.spec, self.device, x, W1t, W2t, idx, offsets, sorted, gate, du)
        dgate = None if gate is None else self.dgate
        _call("more_expert_ffn_backward_ex", self.device, _ptr(x), _ptr(W1t), _ptr(W2t), *self.shape,
              self.addends, _ptr(idx), _ptr(offsets), _ptr(sorted), _ptr(gate), _ptr(du), _ptr(self.dx),
              _ptr(self.dW1t), _ptr(self.dW2t), _ptr(dgate), _ptr(self.workspace), self.workspace_bytes)
        return ExpertGradients(self.dx, self.dW1t, self.dW2t, dgate)


def expert_ffn_backward(x, W1t, W2t, idx, offsets, sorted, gate, du, *, addends: int = 0) -> ExpertGradients:
    """Gradients of expert_ffn given du [T][h] bf16, the gradient with respect to the sum of a token's
    k rows of y; gate may be None (then dgate is None); addends as in expert_ffn (more_expert_ffn_backward_ex)."""
    shape = _ffn_shape(x, W1t, W2t, idx)
    return ExpertFFNBackward(*shape, addends=addends, device=x.device)(x, W1t, W2t, idx, offsets, sorted, gate, du)


# ---------------------------------------------------------------------------------- norms
_RESID_BITS = {torch.float32: 32, torch.bfloat16: 16}


def _resid_bits(dtype) -> int:
    if dtype not in _RESID_BITS:
        raise TypeError("the residual must be float32 or bfloat16, got %s" % dtype)
    return _RESID_BITS[dtype]


@dataclasses.dataclass
class BlockEnd:
    r: torch.Tensor             # [T][h], the new residual (the given one where there is no block)
    xn: Optional[torch.Tensor]  # bfloat16 [T][h], the normed input of the next block
    u: Optional[torch.Tensor]   # bfloat16 [T][h], the block's output summed over its k rows


class BlockNorm:
    """Pre-allocated outputs for repeated block_norm calls with one shape (k = 0: no block, only the
    norm before the first one).  save_u keeps u for the backward pass; inplace writes the new residual
    over the given one."""

    def __init__(self, T: int, h: int, k: int = 1, *, resid_dtype=torch.bfloat16, norm_after: bool = True,
                 alpha: float = 1.0, eps: float = 1e-6, save_u: bool = False, inplace: bool = False, device=None):
        self.shape = (T, h, k)
        for size in (h, k):
            _lib.integer(size, "more_block_norm")
        self.resid_dtype, self.resid_bits = resid_dtype, _resid_bits(resid_dtype)
        self.norm_after, self.alpha, self.eps = bool(norm_after), float(alpha), float(eps)
        self.inplace = inplace
        self.device = dev = _device(device)
        empty = lambda dtype: torch.empty((T, h), dtype=dtype, device=dev)  # noqa: E731
        self.r = empty(resid_dtype) if k > 0 and not inplace else None
        self.u = empty(torch.bfloat16) if k > 0 and save_u else None
        self.xn = empty(torch.bfloat16)

    def __call__(self, r, y=None, *, w_after=None, w_before=None, gate=None) -> BlockEnd:
        T, h, k = self.shape
        dev, f32 = self.device, torch.float32
        if (y is not None) != (k > 0):
            raise ValueError("y must be given exactly when the norm was set up with k > 0")
        _check("r", r, self.resid_dtype, (T, h), dev)
        if y is not None:
            flat = isinstance(y, torch.Tensor) and y.dim() == 2
            _check("y", y, torch.bfloat16, (T * k, h) if flat else (T, k, h), dev)
        if w_after is not None:
            _check("w_after", w_after, f32, (h,), dev)
        if w_before is not None:
            _check("w_before", w_before, f32, (h,), dev)
        if gate is not None:
            _check("gate", gate, f32, (T,), dev)
        out = None if k == 0 else r if self.inplace else self.r
        xn = None if w_before is None else self.xn
        _call("more_block_norm", dev, _ptr(r), self.resid_bits, _ptr(y), T, h, k, _ptr(w_after), _ptr(w_before),
              _ptr(gate), self.alpha, self.eps, int(self.norm_after), _ptr(out), _ptr(self.u), _ptr(xn))
        return BlockEnd(r if out is None else out, xn, self.u)


def block_norm(r, y=None, *, w_after=None, w_before=None, gate=None, norm_after: bool = True, alpha: float = 1.0,
               eps: float = 1e-6, save_u: bool = False) -> BlockEnd:
    """The end of a block and the norm before the next: with u the sum of y's k rows per token
    (y [T k][h] or [T][k][h] bf16) and n = u/rms(u) (or u), r' = alpha r + gate (w_after n) and
    xn = w_before r'/rms(r').  Without y only the norm; without w_before no xn (more_block_norm)."""
    if not isinstance(r, torch.Tensor) or r.dim() != 2:
        raise ValueError("r must be a 2-D tensor")
    if y is not None and (not isinstance(y, torch.Tensor) or y.dim() not in (2, 3)):
        raise ValueError("y must be a 2-D or 3-D tensor")
    T, h = r.shape
    k = 0 if y is None else y.shape[1] if y.dim() == 3 else y.shape[0] // max(T, 1) if T else 1
    call = BlockNorm(T, h, k, resid_dtype=r.dtype, norm_after=norm_after, alpha=alpha, eps=eps, save_u=save_u,
                     device=r.device)
    return call(r, y, w_after=w_after, w_before=w_before, gate=gate)


@dataclasses.dataclass
class BlockEndGradients:
    dr: torch.Tensor                   # [T][h], the residual's type
    du: Optional[torch.Tensor]         # bfloat16 [T][h], the gradient of every row of y
    dw_after: Optional[torch.Tensor]   # float32 [h]
    dw_before: Optional[torch.Tensor]  # float32 [h]
    dgate: Optional[torch.Tensor]      # float32 [T]


def block_norm_backward_workspace_size(T: int, h: int) -> int:
    return _size("more_block_norm_backward_workspace_size", T, h)


class BlockNormBackward:
    """Pre-allocated gradients and workspace for repeated block_norm_backward calls with one shape."""

    def __init__(self, T: int, h: int, *, resid_dtype=torch.bfloat16, norm_after: bool = True, alpha: float = 1.0,
                 eps: float = 1e-6, gated: bool = False, device=None):
        self.shape = (T, h)
        self.resid_dtype, self.resid_bits = resid_dtype, _resid_bits(resid_dtype)
        self.norm_after, self.alpha, self.eps, self.gated = bool(norm_after), float(alpha), float(eps), gated
        self.device = dev = _device(device)
        self.workspace_bytes = block_norm_backward_workspace_size(T, h)
        self.workspace = _workspace(self.workspace_bytes, dev)
        f32 = torch.float32
        self.dr = torch.empty((T, h), dtype=resid_dtype, device=dev)
        self.du = torch.empty((T, h), dtype=torch.bfloat16, device=dev)
        self.dw_after = torch.empty((h,), dtype=f32, device=dev)
        self.dw_before = torch.empty((h,), dtype=f32, device=dev)
        self.dgate = torch.empty((T,), dtype=f32, device=dev) if gated else None

    def __call__(self, u, r_out, dr_out=None, dxn=None, *, dxn32=None, w_after=None, w_before=None,
                 gate=None) -> BlockEndGradients:
        T, h = self.shape
        dev, f32, bf16 = self.device, torch.float32, torch.bfloat16
        if (gate is not None) != self.gated:
            raise ValueError("gate must be given exactly when the backward was set up with gated=True")
        _check("r_out", r_out, self.resid_dtype, (T, h), dev)
        for name, t, dtype, shape in (("u", u, bf16, (T, h)), ("dr_out", dr_out, self.resid_dtype, (T, h)),
                                      ("dxn", dxn, bf16, (T, h)), ("dxn32", dxn32, f32, (T, h)),
                                      ("w_after", w_after, f32, (h,)), ("w_before", w_before, f32, (h,)),
                                      ("gate", gate, f32, (T,))):
            if t is not None:
                _check(name, t, dtype, shape, dev)
        block = u is not None
        du = self.du if block else None
        dwa = self.dw_after if w_after is not None else None
        dwb = self.dw_before if w_before is not None else None
        _call("more_block_norm_backward", dev, _ptr(u), _ptr(r_out), self.resid_bits, _ptr(dr_out), _ptr(dxn),
              _ptr(dxn32), T, h, _ptr(w_after), _ptr(w_before), _ptr(gate), self.alpha, self.eps,
              int(self.norm_after), _ptr(self.dr), _ptr(du), _ptr(dwa), _ptr(dwb), _ptr(self.dgate),
              _ptr(self.workspace), self.workspace_bytes)
        return BlockEndGradients(self.dr, du, dwa, dwb, self.dgate)


def block_norm_backward(u, r_out, dr_out=None, dxn=None, *, dxn32=None, w_after=None, w_before=None, gate=None,
                        norm_after: bool = True, alpha: float = 1.0, eps: float = 1e-6) -> BlockEndGradients:
    """Gradients of block_norm from those of r' (dr_out) and xn (dxn, bf16, plus dxn32, fp32, such as
    the router's dx), given the forward pass's u and r' (u None: no block) (more_block_norm_backward)."""
    if not isinstance(r_out, torch.Tensor) or r_out.dim() != 2:
        raise ValueError("r_out must be a 2-D tensor")
    T, h = r_out.shape
    call = BlockNormBackward(T, h, resid_dtype=r_out.dtype, norm_after=norm_after, alpha=alpha, eps=eps,
                             gated=gate is not None, device=r_out.device)
    return call(u, r_out, dr_out, dxn, dxn32=dxn32, w_after=w_after, w_before=w_before, gate=gate)


# ---------------------------------------------------------------------------------- clipping
class GradClipper:
    """Scales a fixed set of gradients (float32 or bfloat16) to a common 2-norm of at most max_norm:
    by min(1, max_norm / (N + eps)) with N their norm.  In place unless `out` names other tensors.
    `__call__` reads the tensors as they are then and returns (N, the scaled tensors); tensors that have
    been given other storage since are refused."""

    def __init__(self, grads: Sequence[torch.Tensor], max_norm: float, *, eps: float = 1e-6,
                 out: Optional[Sequence[torch.Tensor]] = None):
        grads = list(grads)
        out = grads if out is None else list(out)
        if len(out) != len(grads):
            raise ValueError("out must have as many tensors as grads")
        if not grads:
            raise ValueError("grads is empty")
        for i, (g, o) in enumerate(zip(grads, out)):
            if not isinstance(g, torch.Tensor) or not isinstance(o, torch.Tensor):
                raise TypeError("gradients must be torch.Tensors")
            if g.dtype not in _RESID_BITS:
                raise TypeError("gradient %d must be float32 or bfloat16, got %s" % (i, g.dtype))
            if not g.is_contiguous():
                raise ValueError("gradient %d must be contiguous" % i)
            if g.device.type != "cuda":
                raise ValueError("gradient %d must be on a GPU device" % i)
            _check("out[%d]" % i, o, g.dtype, g.shape, grads[0].device)
            if g.device != grads[0].device:
                raise ValueError("gradients must be on one device")
        # an output may be its own input, and may overlap nothing else
        spans = [(o.data_ptr(), o.data_ptr() + o.numel() * o.element_size(), True, "out[%d]" % i)
                 for i, o in enumerate(out) if o.numel()]
        spans += [(g.data_ptr(), g.data_ptr() + g.numel() * g.element_size(), False, "grads[%d]" % i)
                  for i, (g, o) in enumerate(zip(grads, out)) if g.numel() and g.data_ptr() != o.data_ptr()]
        ends = {True: (0, ""), False: (0, "")}  # of the outputs and inputs seen so far, by address
        for start, end, is_out, name in sorted(spans):
            for other in (True, False):
                if (is_out or other) and start < ends[other][0]:
                    raise ValueError("%s overlaps %s" % (name, ends[other][1]))
            ends[is_out] = max(ends[is_out], (end, name))
        self.grads, self.out = grads, out
        self.max_norm, self.eps = float(max_norm), float(eps)
        self.device = grads[0].device
        n = len(grads)
        self._tensors = grads if all(g is o for g, o in zip(grads, out)) else grads + out
        self._places = list(map(torch.Tensor.data_ptr, self._tensors))
        self._in = (ctypes.c_void_p * n)(*self._places[:n])
        self._out = (ctypes.c_void_p * n)(*self._places[-n:])
        self._numel = (ctypes.c_int64 * n)(*[g.numel() for g in grads])
        self._bits = (ctypes.c_int32 * n)(*[_RESID_BITS[g.dtype] for g in grads])
        self.workspace_bytes = _size("more_grad_clip_workspace_size", self._numel, n)
        self.workspace = _workspace(self.workspace_bytes, self.device)
        self.norm = torch.empty((), dtype=torch.float32, device=self.device)

    def __call__(self):
        if list(map(torch.Tensor.data_ptr, self._tensors)) != self._places:
            raise ValueError("a tensor's storage has changed since the clipper was set up")
        _call("more_grad_clip", self.device, self._in, self._out, self._numel, self._bits, len(self.grads),
              self.max_norm, self.eps, _ptr(self.norm), _ptr(self.workspace), self.workspace_bytes)
        return self.norm, self.out


def clip_gradients(grads: Sequence[torch.Tensor], max_norm: float, *, eps: float = 1e-6) -> torch.Tensor:
    """Scales the gradients in place to a common 2-norm of at most max_norm; returns the norm that they
    had (a float32 scalar on their device)."""
    return GradClipper(grads, max_norm, eps=eps)()[0]
