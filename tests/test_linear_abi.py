"""The C ABI and the binding of the linear maps, the quantisation and the distillation on the host: refusals and size
queries (no GPU needed: every call fails validation or is a host query)."""
import ctypes
import os

import pytest

from paper_2609_36301_amd import _lib

FAKE = ctypes.c_void_p(0x10000)  # aligned, never dereferenced (validation fails first)
ODD = ctypes.c_void_p(0x10002)
BYTE = ctypes.c_void_p(0x10001)
HALF = ctypes.c_void_p(0x10008)  # 8-byte aligned
INVALID, UNSUPPORTED, WORKSPACE = _lib.ERR_INVALID_ARG, _lib.ERR_UNSUPPORTED, _lib.ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2609_36301_amd import build
        build.build(verbose=False)
    return _lib.load()


BIG = dict(T=4096, K=512, N=512, M=4096, k=2)  # listed tiles: a workspace is needed


def linear(lib, T=64, K=64, N=16, M=8, k=2, x=FAKE, W=FAKE, idx=FAKE, offsets=FAKE, srt=FAKE, y=FAKE, bits=16, ws=None, wsb=0):
    return lib.more_expert_linear(x, W, T, K, N, M, k, idx, offsets, srt, y, bits, ws, wsb, None)


def backward(lib, T=64, K=64, N=16, M=8, k=2, x=FAKE, W=FAKE, idx=FAKE, offsets=FAKE, srt=FAKE, dy=FAKE, dx=FAKE, dW=FAKE,
             ws=None, wsb=0):
    return lib.more_expert_linear_backward(x, W, T, K, N, M, k, idx, offsets, srt, dy, dx, dW, ws, wsb, None)


def q8(lib, T=64, K=64, N=16, M=8, k=2, x=FAKE, qs=FAKE, W=FAKE, wsc=FAKE, idx=FAKE, offsets=FAKE, srt=FAKE, gate=FAKE, y=FAKE,
       bits=16, ws=None, wsb=0):
    return lib.more_expert_linear_q8(x, qs, W, wsc, T, K, N, M, k, idx, offsets, srt, gate, y, bits, ws, wsb, None)


SHAPES = [(dict(T=-1), INVALID), (dict(K=0), INVALID), (dict(N=0), INVALID), (dict(M=0), INVALID), (dict(k=0), INVALID),
          (dict(K=68), UNSUPPORTED), (dict(N=12), UNSUPPORTED), (dict(k=33), UNSUPPORTED), (dict(M=1 << 30), UNSUPPORTED),
          (dict(T=1 << 30), UNSUPPORTED), (dict(K=65552), UNSUPPORTED), (dict(N=(1 << 20) + 8), UNSUPPORTED)]
POINTERS = [(dict(**{name: value}), INVALID) for name in ("x", "W", "idx", "offsets", "srt") for value in (None, BYTE)]
POINTERS += [(dict(x=HALF), INVALID), (dict(W=HALF), INVALID), (dict(idx=ODD), INVALID)]


@pytest.mark.parametrize("kw,status", SHAPES + POINTERS + [(dict(y=None), INVALID), (dict(y=HALF), INVALID), (dict(bits=8), INVALID),
                                                          (dict(ws=HALF, wsb=1 << 30), INVALID), (BIG, WORKSPACE),
                                                          (dict(BIG, ws=FAKE, wsb=16), WORKSPACE)])
def test_linear_refusals(lib, kw, status):
    assert linear(lib, **kw) == status


@pytest.mark.parametrize("kw,status", SHAPES + POINTERS + [
    (dict(dy=None), INVALID), (dict(dy=HALF), INVALID), (dict(dx=None, dW=None), INVALID), (dict(dx=HALF), INVALID),
    (dict(dW=HALF), INVALID), ({}, WORKSPACE), (dict(dx=None), WORKSPACE), (dict(dW=None), WORKSPACE),
    (dict(ws=FAKE, wsb=16), WORKSPACE)])
def test_backward_refusals(lib, kw, status):
    assert backward(lib, **kw) == status


@pytest.mark.parametrize("kw,status", SHAPES + POINTERS + [
    (dict(K=72), UNSUPPORTED), (dict(K=-16), INVALID), (dict(y=None), INVALID), (dict(bits=64), INVALID), (dict(qs=None), INVALID),
    (dict(qs=ODD), INVALID), (dict(wsc=None), INVALID), (dict(wsc=HALF), INVALID), (dict(gate=ODD), INVALID), (BIG, WORKSPACE)])
def test_q8_refusals(lib, kw, status):
    assert q8(lib, **kw) == status


def quantize(lib, x=FAKE, T=4, width=64, gated=0, q=FAKE, scale=FAKE):
    return lib.more_quantize_rows(x, T, width, gated, q, scale, None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), INVALID), (dict(width=0), INVALID), (dict(width=24), UNSUPPORTED), (dict(width=65552), UNSUPPORTED),
    (dict(T=1 << 31), UNSUPPORTED), (dict(x=None), INVALID), (dict(q=None), INVALID), (dict(scale=None), INVALID),
    (dict(x=HALF), INVALID), (dict(q=HALF), INVALID), (dict(scale=ODD), INVALID), (dict(T=0, x=None, q=None, scale=None), _lib.OK)])
def test_quantize_refusals(lib, kw, status):
    assert quantize(lib, **kw) == status


def distill(lib, z=FAKE, bits=32, T=4, V=50, ld=50, ids=FAKE, values=FAKE, k=3, tau=1.0, weight=FAKE, loss=FAKE, m=FAKE, Z=FAKE,
            d=HALF, ldd=50):
    return lib.more_distill(z, bits, T, V, ld, ids, values, k, tau, weight, loss, m, Z, d, ldd, None)


def distill_backward(lib, z=FAKE, bits=32, T=4, V=50, ld=50, ids=FAKE, values=FAKE, k=3, tau=1.0, weight=FAKE, m=FAKE, Z=FAKE,
                     d=HALF, ldd=50):
    return lib.more_distill_backward(z, bits, T, V, ld, m, Z, ids, values, k, tau, weight, d, ldd, None)


BOTH = [(dict(T=-1), INVALID), (dict(V=0), INVALID), (dict(k=0), INVALID), (dict(bits=8), INVALID), (dict(tau=0.0), INVALID),
        (dict(tau=-1.0), INVALID), (dict(tau=float("nan")), INVALID), (dict(tau=float("inf")), INVALID), (dict(ld=49), INVALID),
        (dict(ldd=49), INVALID), (dict(z=None), INVALID), (dict(ids=None), INVALID), (dict(values=None), INVALID),
        (dict(z=ODD), INVALID), (dict(z=BYTE, bits=16), INVALID), (dict(ids=ODD), INVALID), (dict(values=ODD), INVALID),
        (dict(weight=ODD), INVALID), (dict(m=ODD), INVALID), (dict(Z=ODD), INVALID), (dict(d=ODD), INVALID),
        (dict(d=FAKE, ldd=64), INVALID),  # in place with another stride
        (dict(V=(1 << 30) + 1, ld=1 << 31, ldd=1 << 31), UNSUPPORTED), (dict(k=1025), UNSUPPORTED), (dict(T=1 << 31), UNSUPPORTED),
        (dict(tau=2.0 ** -41), UNSUPPORTED), (dict(tau=1e-45), UNSUPPORTED), (dict(tau=2.0 ** 41), UNSUPPORTED),
        (dict(ld=(1 << 40) + 1), UNSUPPORTED), (dict(ldd=(1 << 40) + 1), UNSUPPORTED),
        (dict(T=0, z=None, ids=None, values=None), _lib.OK)]


@pytest.mark.parametrize("kw,status", BOTH + [(dict(loss=ODD), INVALID), (dict(loss=None, m=None, Z=None, d=None), INVALID)])
def test_distill_refusals(lib, kw, status):
    assert distill(lib, **kw) == status


@pytest.mark.parametrize("kw,status", BOTH + [(dict(m=None), INVALID), (dict(Z=None), INVALID), (dict(weight=None), INVALID),
                                              (dict(d=None), INVALID)])
def test_distill_backward_refusals(lib, kw, status):
    assert distill_backward(lib, **kw) == status


def test_sizes_and_plans(lib):
    n = ctypes.c_size_t(0)
    most = (1 << 31) - (1 << 16)
    for f in (lib.more_expert_linear_workspace_size, lib.more_expert_linear_backward_workspace_size,
              lib.more_expert_linear_q8_workspace_size):
        assert f(most, 16, 8, 2, 1, ctypes.byref(n)) == _lib.OK
        assert f(most + 1, 16, 8, 2, 1, ctypes.byref(n)) == UNSUPPORTED
        assert f(most // 32 + 1, 16, 8, 2, 32, ctypes.byref(n)) == UNSUPPORTED
        assert f(0, 64, 64, 8, 2, ctypes.byref(n)) == _lib.OK and n.value == 0
        assert f(4, 64, 64, 8, 2, None) == INVALID
        assert f(4096, 65536, 1 << 20, 3, 1, ctypes.byref(n)) == _lib.OK
    plan = _lib.LinearPlan()
    for kind, status in ((-1, INVALID), (3, INVALID), (0, _lib.OK), (1, _lib.OK), (2, _lib.OK)):
        assert lib.more_expert_linear_plan(64, 64, 64, 8, 2, kind, ctypes.byref(plan)) == status
    assert lib.more_expert_linear_plan(64, 64, 64, 8, 2, 0, None) == INVALID
    assert lib.more_expert_linear_plan(64, 72, 64, 8, 2, 2, ctypes.byref(plan)) == UNSUPPORTED


def test_binding_refuses_before_the_gpu():
    torch = pytest.importorskip("torch")
    import paper_2609_36301_amd as more
    from paper_2609_36301_amd import distill as d, linear as m
    z = torch.zeros
    with pytest.raises(ValueError, match="x must have 2 dimensions"):
        more.expert_linear(z(4), z(2, 8, 8), z(4, 1), z(3), z(4))
    with pytest.raises(TypeError, match="Wq must be a torch.Tensor"):
        more.expert_linear_q8(z(4, 16), z(4), None, z(2, 8), z(4, 1), z(3), z(4))
    with pytest.raises(TypeError, match="output must be bfloat16 or float32"):
        m.ExpertLinear(4, 8, 8, 2, 1, out_dtype=torch.float16)
    with pytest.raises(ValueError, match="need_dx or need_dW"):
        m.ExpertLinearBackward(4, 8, 8, 2, 1, need_dx=False, need_dW=False)
    with pytest.raises(TypeError, match="x must be a torch.Tensor"):
        more.quantize_rows([[1.0]])
    with pytest.raises(ValueError, match="contiguous"):
        more.quantize_rows(z(32, 16, dtype=torch.bfloat16).t())
    with pytest.raises(ValueError, match="even number"):
        more.quantize_rows(z(4, 17, dtype=torch.bfloat16), gated=True)
    with pytest.raises(ValueError, match="GPU"):
        more.quantize_rows(z(4, 16, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="logits must be a 2-D tensor"):
        more.distill_loss(z(4), z(4, 2), z(4, 2))
    with pytest.raises(ValueError, match="must not overlap"):
        more.distill_loss(z(1, 8).expand(4, 8), z(4, 2), z(4, 2))
    with pytest.raises(TypeError, match="logits must be float32 or bfloat16"):
        more.distill_loss(z(4, 8, dtype=torch.float16), z(4, 2), z(4, 2))
    with pytest.raises(ValueError, match="ld must be at least"):
        d.Distill(4, 8, 2, ld=7)
    with pytest.raises(ValueError, match="teacher_idx must be a 2-D tensor"):
        more.distill_backward(z(4, 8), z(4), z(4), z(4), z(4, 2), z(4))
