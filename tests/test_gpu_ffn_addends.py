"""Two bf16 addends between the experts' products at every size, on request: the results keep the bounds without the
rounding of the hidden units and of their gradients to one bf16 (layer_ref.py with planes=2), on tiles of every size
(values marked `gpu`; plans and refusals on the host)."""
import ctypes

import numpy as np
import pytest

import layer_ref as ref
from gpu_util import announce, require_gpu
from test_gpu_ffn import check, make, on_device
from test_layer_abi import lib  # noqa: F401

# more values than 2^15, which the library itself carries as one addend: (shape, rows of a tile forward and backward)
SHAPES = {
    "tiles_of_32": (dict(T=500, h=1040, s=40, M=150, k=3, drop=0.1), 32, 32),
    "tiles_of_32_long_spans": (dict(T=4336, h=704, s=80, M=396, k=1, drop=0.02), 32, 32),
    "tiles_of_64": (dict(T=900, h=144, s=136, M=16, k=3, hot=0.6, drop=0.03), 64, 64),
    "tiles_of_64_long_spans": (dict(T=6000, h=2064, s=40, M=128, k=1), 64, 64),
    "tiles_of_128": (dict(T=8000, h=48, s=136, M=128, k=1, drop=0.01), 128, 128),
    "tiles_of_256": (dict(T=16000, h=496, s=200, M=32, k=1, hot=0.4), 256, 128),
    "large_weight_gradient_tiles": (dict(T=218, h=656, s=264, M=290, k=1), 32, 32),
    "runs": (dict(T=2500, h=528, s=264, M=4, k=1, hot=0.5, drop=0.02), 64, 64),
    "dense": (dict(T=1100, h=80, s=40, M=1, k=1, gated=False), 0, 64),
}


def _plans(kw, **more):
    from paper_2609_36301_amd import expert_ffn_plan
    return [expert_ffn_plan(kw["T"], kw["h"], kw["s"], kw["M"], kw["k"], backward=b, **more) for b in (False, True)]


@pytest.mark.parametrize("name", list(SHAPES))
def test_plan(name):
    kw, *rows = SHAPES[name]
    assert kw["T"] * kw["k"] * kw["s"] > 2 ** 15
    plain, two = _plans(kw), _plans(kw, addends=2)
    assert [p["addends"] for p in plain] == [1 if rows[0] else 2, 1]
    assert [p["addends"] for p in two] == [2, 2] and [p["tile_rows"] for p in two] == rows
    from paper_2609_36301_amd import layer
    shape = [kw[n] for n in ("T", "h", "s", "M", "k")]
    hidden = kw["T"] * kw["k"] * kw["s"] * 2
    if rows[0]:  # (parts of a workspace are rounded up to 256 bytes)
        assert layer.expert_ffn_workspace_size(*shape, addends=2) > layer.expert_ffn_workspace_size(*shape) + hidden - 256
    assert layer.expert_ffn_backward_workspace_size(*shape, addends=2) >= 6 * hidden + kw["T"] * kw["k"] * kw["h"] * 4


@pytest.mark.parametrize("addends", [-1, 1, 3])
def test_refusals(lib, addends):  # noqa: F811
    from paper_2609_36301_amd import _lib, layer
    n, fake = ctypes.c_size_t(0), ctypes.c_void_p(0x10000)
    for size in (lib.more_expert_ffn_workspace_size_ex, lib.more_expert_ffn_backward_workspace_size_ex):
        assert size(64, 64, 16, 8, 2, addends, ctypes.byref(n)) == _lib.ERR_INVALID_ARG
    assert lib.more_expert_ffn_plan(64, 64, 16, 8, 2, addends, 0, ctypes.byref(_lib.ExpertPlan())) == _lib.ERR_INVALID_ARG
    assert lib.more_expert_ffn_ex(fake, fake, fake, 64, 64, 16, 8, 2, addends, fake, fake, fake, fake, fake, fake, 1 << 40,
                                  None) == _lib.ERR_INVALID_ARG
    assert lib.more_expert_ffn_backward_ex(fake, fake, fake, 64, 64, 16, 8, 2, addends, fake, fake, fake, fake, fake, fake,
                                           fake, fake, fake, fake, 1 << 40, None) == _lib.ERR_INVALID_ARG
    with pytest.raises(_lib.MoreError):
        layer.expert_ffn_workspace_size(64, 64, 16, 8, 2, addends)


def test_workspace_of_two_addends_is_checked(lib):  # noqa: F811
    from paper_2609_36301_amd import _lib
    fake, plain, two = ctypes.c_void_p(0x10000), ctypes.c_size_t(0), ctypes.c_size_t(0)
    shape = (500, 1040, 40, 150, 3)
    assert lib.more_expert_ffn_workspace_size_ex(*shape, 0, ctypes.byref(plain)) == _lib.OK
    assert lib.more_expert_ffn_workspace_size_ex(*shape, 2, ctypes.byref(two)) == _lib.OK and two.value > plain.value
    assert lib.more_expert_ffn_ex(fake, fake, fake, *shape, 2, fake, fake, fake, fake, fake, fake, plain.value,
                                  None) == _lib.ERR_WORKSPACE
    assert lib.more_expert_ffn_backward_workspace_size_ex(*shape, 0, ctypes.byref(plain)) == _lib.OK
    assert lib.more_expert_ffn_backward_ex(fake, fake, fake, *shape, 2, fake, fake, fake, fake, fake, fake, fake, fake, fake,
                                           fake, plain.value, None) == _lib.ERR_WORKSPACE


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(SHAPES))
def test_values(name):
    kw = SHAPES[name][0]
    M = kw["M"]
    idx, bits, gate, exact = make(**kw, seed=21)
    torch = require_gpu()
    from paper_2609_36301_amd import layer
    announce("expert_ffn and its backward pass with two addends, %s %s" % (name, kw))
    d, i, o, s, g = on_device(idx, bits, gate, M)
    y = layer.expert_ffn(d["x"], d["W1t"], d["W2t"], i, o, s, g, addends=2)
    got = layer.expert_ffn_backward(d["x"], d["W1t"], d["W2t"], i, o, s, g, d["du"], addends=2)
    torch.cuda.synchronize()
    given = (exact["x"], exact["W1t"], exact["W2t"], idx, exact["gate"])
    want, bound = ref.ffn(*given, planes=2)
    check("y", y.float().cpu().numpy(), want, bound, name)
    want, bound = ref.ffn_backward(*given, exact["du"], planes=2)
    for field, v, b in zip(("dx", "dW1t", "dW2t", "dgate"), want, bound):
        if getattr(got, field) is not None:
            check(field, getattr(got, field).float().cpu().numpy(), v, b, name)


@pytest.mark.gpu
def test_calls_without_the_choice_are_those_of_zero():
    """more_expert_ffn and its backward pass, as C programs call them, against the binding's calls, bit for bit."""
    torch = require_gpu()
    from paper_2609_36301_amd import _lib, layer
    kw, *_ = SHAPES["tiles_of_64"]
    shape = [kw[n] for n in ("T", "h", "s", "M", "k")]
    idx, bits, gate, _ = make(**kw)
    d, i, o, s, g = on_device(idx, bits, gate, kw["M"])
    announce("more_expert_ffn and more_expert_ffn_backward %s" % kw)
    want = layer.expert_ffn(d["x"], d["W1t"], d["W2t"], i, o, s, g)
    grads = layer.expert_ffn_backward(d["x"], d["W1t"], d["W2t"], i, o, s, g, d["du"])
    lib, stream, n = _lib.load(), torch.cuda.current_stream().cuda_stream, ctypes.c_size_t(0)
    p = lambda t: t.data_ptr()  # noqa: E731
    _lib.check(lib.more_expert_ffn_workspace_size(*shape, ctypes.byref(n)), "size")
    y, ws = torch.empty_like(want), torch.empty(n.value, dtype=torch.uint8, device="cuda")
    _lib.check(lib.more_expert_ffn(p(d["x"]), p(d["W1t"]), p(d["W2t"]), *shape, p(i), p(o), p(s), p(g), p(y), p(ws), n.value,
                                   stream), "more_expert_ffn")
    _lib.check(lib.more_expert_ffn_backward_workspace_size(*shape, ctypes.byref(n)), "size")
    out, ws2 = [torch.empty_like(t) for t in (grads.dx, grads.dW1t, grads.dW2t, grads.dgate)], torch.empty(
        n.value, dtype=torch.uint8, device="cuda")
    _lib.check(lib.more_expert_ffn_backward(p(d["x"]), p(d["W1t"]), p(d["W2t"]), *shape, p(i), p(o), p(s), p(g), p(d["du"]),
                                            *map(p, out), p(ws2), n.value, stream), "more_expert_ffn_backward")
    torch.cuda.synchronize()
    assert torch.equal(y, want)
    for a, b in zip(out, (grads.dx, grads.dW1t, grads.dW2t, grads.dgate)):
        assert torch.equal(a, b)
    assert np.isfinite(y.float().cpu().numpy()).all()
