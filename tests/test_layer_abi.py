"""The C ABI and the binding of the layer's operators on the host: refusals and size queries (no GPU
needed: every call fails validation or is a host query)."""
import ctypes
import os

import pytest

from paper_2609_36301_amd import _lib

FAKE = ctypes.c_void_p(0x10000)  # aligned, never dereferenced (validation fails first)
ODD = ctypes.c_void_p(0x10002)
HALF = ctypes.c_void_p(0x10008)  # 8-byte aligned
INVALID, UNSUPPORTED, WORKSPACE = _lib.ERR_INVALID_ARG, _lib.ERR_UNSUPPORTED, _lib.ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2609_36301_amd import build
        build.build(verbose=False)
    return _lib.load()


def ffn(lib, T=64, h=64, s=16, M=8, k=2, x=FAKE, W1t=FAKE, W2t=FAKE, idx=FAKE, offsets=FAKE, srt=FAKE, gate=FAKE,
        y=FAKE, ws=None, wsb=0):
    return lib.more_expert_ffn(x, W1t, W2t, T, h, s, M, k, idx, offsets, srt, gate, y, ws, wsb, None)


def ffn_backward(lib, T=64, h=64, s=16, M=8, k=2, x=FAKE, W1t=FAKE, W2t=FAKE, idx=FAKE, offsets=FAKE, srt=FAKE,
                 gate=FAKE, du=FAKE, dx=FAKE, dW1t=FAKE, dW2t=FAKE, dgate=FAKE, ws=None, wsb=0):
    return lib.more_expert_ffn_backward(x, W1t, W2t, T, h, s, M, k, idx, offsets, srt, gate, du, dx, dW1t, dW2t,
                                        dgate, ws, wsb, None)


SHAPES = [(dict(T=-1), INVALID), (dict(h=0), INVALID), (dict(s=0), INVALID), (dict(M=0), INVALID), (dict(k=0), INVALID),
          (dict(h=72), UNSUPPORTED), (dict(s=12), UNSUPPORTED), (dict(k=33), UNSUPPORTED), (dict(M=1 << 30), UNSUPPORTED),
          (dict(T=1 << 30), UNSUPPORTED), (dict(h=65552), UNSUPPORTED), (dict(s=65544), UNSUPPORTED)]
POINTERS = [(dict(**{name: value}), INVALID) for name in ("x", "W1t", "W2t", "idx", "offsets", "srt")
            for value in (None, ODD)] + [(dict(W1t=HALF), INVALID), (dict(gate=ODD), INVALID)]


@pytest.mark.parametrize("kw,status", SHAPES + POINTERS + [(dict(y=None), INVALID), (dict(y=HALF), INVALID), ({}, WORKSPACE)])
def test_ffn_refusals(lib, kw, status):
    assert ffn(lib, **kw) == status


@pytest.mark.parametrize("kw,status", SHAPES + POINTERS + [
    (dict(**{name: value}), INVALID) for name in ("du", "dx", "dW1t", "dW2t") for value in (None, HALF)] + [
    (dict(gate=None), INVALID), (dict(dgate=ODD), INVALID), ({}, WORKSPACE)])
def test_ffn_backward_refusals(lib, kw, status):
    assert ffn_backward(lib, **kw) == status


def test_ffn_workspace(lib):
    n, m = ctypes.c_size_t(0), ctypes.c_size_t(0)
    size, back = lib.more_expert_ffn_workspace_size, lib.more_expert_ffn_backward_workspace_size
    assert size(64, 64, 16, 8, 2, ctypes.byref(n)) == _lib.OK and n.value >= 64 * 2 * 16 * 2
    assert ffn(lib, ws=FAKE, wsb=n.value - 1) == WORKSPACE
    assert ffn(lib, ws=ctypes.c_void_p(0x10010), wsb=n.value) == INVALID  # 256-byte alignment
    assert back(64, 64, 16, 8, 2, ctypes.byref(m)) == _lib.OK and m.value > n.value
    assert ffn_backward(lib, ws=FAKE, wsb=m.value - 1) == WORKSPACE
    for f in (size, back):
        assert f(0, 64, 16, 8, 2, ctypes.byref(n)) == _lib.OK and n.value == 0
        assert f(64, 64, 16, 8, 2, None) == INVALID
        assert f(64, 60, 16, 8, 2, ctypes.byref(n)) == UNSUPPORTED
    # an empty batch launches nothing, and its token-sized buffers may be NULL
    assert ffn(lib, T=0, x=None, idx=None, srt=None, y=None) == _lib.OK
    assert ffn(lib, T=0, offsets=None) == INVALID


def norm(lib, r=FAKE, bits=16, y=FAKE, T=4, h=64, k=2, w_after=FAKE, w_before=FAKE, gate=FAKE, alpha=1.0, eps=1e-6,
         after=1, r_out=FAKE, u=FAKE, xn=FAKE):
    return lib.more_block_norm(r, bits, y, T, h, k, w_after, w_before, gate, alpha, eps, after, r_out, u, xn, None)


@pytest.mark.parametrize("kw,status", [
    (dict(r=None), INVALID), (dict(y=None), INVALID), (dict(r_out=None), INVALID), (dict(xn=None), INVALID),
    (dict(w_before=None), INVALID), (dict(bits=8), INVALID), (dict(T=-1), INVALID), (dict(h=0), INVALID),
    (dict(k=-1), INVALID), (dict(k=0), INVALID), (dict(k=0, y=None, w_after=None, gate=None, u=None), INVALID),
    (dict(k=0, y=None, w_after=None, gate=None, u=None, r_out=None, w_before=None, xn=None), INVALID),
    (dict(eps=0.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(alpha=float("inf")), INVALID),
    (dict(h=72), UNSUPPORTED), (dict(h=_lib.NORM_H_MAX + 16), UNSUPPORTED), (dict(T=1 << 31), UNSUPPORTED),
    (dict(k=65537), UNSUPPORTED), (dict(T=1 << 30, k=2), UNSUPPORTED),
    (dict(r=HALF), INVALID), (dict(y=HALF), INVALID), (dict(w_after=HALF), INVALID), (dict(w_before=HALF), INVALID),
    (dict(gate=ODD), INVALID), (dict(r_out=HALF), INVALID), (dict(u=HALF), INVALID), (dict(xn=HALF), INVALID),
    (dict(T=0, r=None, y=None, r_out=None, u=None, xn=None, gate=None), _lib.OK)])
def test_norm_refusals(lib, kw, status):
    assert norm(lib, **kw) == status


def norm_backward(lib, u=FAKE, r_out=FAKE, bits=16, dr_out=FAKE, dxn=FAKE, dxn32=FAKE, T=4, h=64, w_after=FAKE,
                  w_before=FAKE, gate=FAKE, alpha=1.0, eps=1e-6, after=1, dr=FAKE, du=FAKE, dwa=FAKE, dwb=FAKE,
                  dgate=FAKE, ws=None, wsb=0):
    return lib.more_block_norm_backward(u, r_out, bits, dr_out, dxn, dxn32, T, h, w_after, w_before, gate, alpha, eps,
                                        after, dr, du, dwa, dwb, dgate, ws, wsb, None)


@pytest.mark.parametrize("kw,status", [
    (dict(r_out=None), INVALID), (dict(dr=None), INVALID), (dict(du=None), INVALID), (dict(u=None), INVALID),
    (dict(gate=None), INVALID), (dict(w_before=None), INVALID), (dict(w_before=None, dwb=None), INVALID),
    (dict(dxn=None, dxn32=None), INVALID), (dict(dr_out=None, dxn=None, dxn32=None, w_before=None, dwb=None), INVALID),
    (dict(bits=64), INVALID), (dict(eps=-1.0), INVALID), (dict(h=40), UNSUPPORTED), (dict(h=8208), UNSUPPORTED),
    (dict(u=HALF), INVALID), (dict(dxn=HALF), INVALID), (dict(dxn32=HALF), INVALID), (dict(dr=HALF), INVALID),
    (dict(dwa=ODD), INVALID), (dict(dgate=ODD), INVALID), ({}, WORKSPACE), (dict(ws=FAKE, wsb=4), WORKSPACE),
    (dict(u=None, w_after=None, gate=None, du=None, dwa=None, dgate=None), WORKSPACE)])
def test_norm_backward_refusals(lib, kw, status):
    assert norm_backward(lib, **kw) == status


def test_norm_backward_workspace(lib):
    n = ctypes.c_size_t(0)
    assert lib.more_block_norm_backward_workspace_size(100, 64, ctypes.byref(n)) == _lib.OK and n.value > 0
    assert lib.more_block_norm_backward_workspace_size(0, 64, ctypes.byref(n)) == _lib.OK and n.value == 0
    assert lib.more_block_norm_backward_workspace_size(100, 64, None) == INVALID


def grad_clip(lib, ptrs=(0x10000, 0x20000), outs=None, numel=(4, 5), bits=(32, 16), max_norm=1.0, eps=1e-6, norm=FAKE,
              ws=FAKE, wsb=1 << 20, n=None):
    outs = ptrs if outs is None else outs
    c = len(ptrs)
    return lib.more_grad_clip((ctypes.c_void_p * c)(*ptrs), (ctypes.c_void_p * c)(*outs), (ctypes.c_int64 * c)(*numel),
                              (ctypes.c_int32 * c)(*bits), c if n is None else n, max_norm, eps, norm, ws, wsb, None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), INVALID), (dict(numel=(4, -1)), INVALID), (dict(numel=(4, 1 << 41)), UNSUPPORTED),
    (dict(bits=(32, 8)), INVALID), (dict(ptrs=(0, 0x20000)), INVALID), (dict(ptrs=(0x10002, 0x20000)), INVALID),
    (dict(ptrs=(0x10000, 0x20001)), INVALID), (dict(outs=(0x10000, 0)), INVALID), (dict(max_norm=-1.0), INVALID),
    (dict(max_norm=float("nan")), INVALID), (dict(max_norm=float("inf")), INVALID), (dict(eps=0.0), INVALID),
    (dict(norm=ODD), INVALID), (dict(ws=HALF), INVALID), (dict(ws=None), WORKSPACE), (dict(wsb=0), WORKSPACE)])
def test_clip_refusals(lib, kw, status):
    assert grad_clip(lib, **kw) == status


def test_clip_null_arrays(lib):
    assert lib.more_grad_clip(None, None, None, None, 2, 1.0, 1e-6, FAKE, FAKE, 1 << 20, None) == INVALID
    assert lib.more_grad_clip_workspace_size(None, 1, ctypes.byref(ctypes.c_size_t(0))) == INVALID


def test_binding_refuses_what_is_not_on_a_gpu():
    torch = pytest.importorskip("torch")
    from paper_2609_36301_amd import layer
    with pytest.raises(ValueError, match="GPU"):
        layer._device("cpu")
    with pytest.raises(ValueError, match="GPU"):
        layer.clip_gradients([torch.zeros(4)], 1.0)
    with pytest.raises(ValueError, match="empty"):
        layer.GradClipper([], 1.0)
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        layer.GradClipper([torch.zeros(4, dtype=torch.float64)], 1.0)
    with pytest.raises(TypeError, match="residual"):
        layer.BlockNorm(4, 64, 1, resid_dtype=torch.float16)


def test_ffn_most_entries(lib):
    """The kernels add up to a tile's rows to an entry in 32 bits, so 2^16 entries are kept free."""
    n = ctypes.c_size_t(0)
    most = (1 << 31) - (1 << 16)
    for f in (lib.more_expert_ffn_workspace_size, lib.more_expert_ffn_backward_workspace_size):
        assert f(most, 16, 8, 2, 1, ctypes.byref(n)) == _lib.OK and n.value >= most * 16
        assert f(most + 1, 16, 8, 2, 1, ctypes.byref(n)) == UNSUPPORTED
        assert f(most // 32 + 1, 16, 8, 2, 32, ctypes.byref(n)) == UNSUPPORTED


def test_block_norm_refuses_before_the_gpu():
    torch = pytest.importorskip("torch")
    from paper_2609_36301_amd import block_norm
    r = torch.zeros((4, 64))
    for y in (torch.zeros(64), torch.zeros((1, 4, 2, 64)), [[0.0] * 64]):
        with pytest.raises(ValueError, match="y must be a 2-D or 3-D tensor"):
            block_norm(r, y)
