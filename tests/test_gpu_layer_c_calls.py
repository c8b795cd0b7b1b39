"""Calls that include/more.h allows and the binding does not make: outputs left out, outputs over their inputs, no
tensors, no tokens (marked `gpu`)."""
import ctypes

import numpy as np
import pytest

import layer_ref as ref
from gpu_util import announce, require_gpu
from test_gpu_block_norm import _case, _dev, _f64
from test_gpu_ffn import CASES, check, make, on_device

pytestmark = pytest.mark.gpu


def _p(t):
    return None if t is None else t.data_ptr()


def _lib():
    torch = require_gpu()
    from paper_2609_36301_amd import _lib
    return torch, _lib.load(), _lib.check, torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("h,bits", [(272, 32), (1040, 16), (4112, 32)])
def test_norm_backward_in_place_and_without_some_outputs(h, bits):
    torch, lib, ok, stream = _lib()
    from paper_2609_36301_amd import layer
    T, eps = 1500, 1e-3
    a = _case(T, h, 1, bits, True, seed=31)
    d, e = _dev(a), {n: _f64(v) for n, v in a.items()}
    announce("more_block_norm_backward, dr over dr_out, T=%d h=%d" % (T, h))
    want = layer.block_norm_backward(d["u"], d["r"], d["dr_out"], d["dxn"], w_after=d["w_after"], w_before=d["w_before"],
                                     gate=d["gate"], alpha=0.75, eps=eps)
    ws = torch.empty(layer.block_norm_backward_workspace_size(T, h), dtype=torch.uint8, device="cuda")

    def call(w_after, dwa, dwb, dgate):
        dr, du = d["dr_out"].clone(), torch.empty((T, h), dtype=torch.bfloat16, device="cuda")
        ok(lib.more_block_norm_backward(_p(d["u"]), _p(d["r"]), bits, _p(dr), _p(d["dxn"]), None, T, h, _p(w_after),
                                        _p(d["w_before"]), _p(d["gate"]), 0.75, eps, 1, _p(dr), _p(du), _p(dwa), _p(dwb),
                                        _p(dgate), _p(ws), ws.numel(), stream), "more_block_norm_backward")
        return dr, du

    dr, du = call(d["w_after"], None, None, None)
    assert torch.equal(dr, want.dr) and torch.equal(du, want.du)
    dwb = torch.empty(h, device="cuda")
    call(d["w_after"], None, dwb, None)
    assert torch.equal(dwb, want.dw_before)
    # a weight of ones that is not passed has a gradient too
    dwa = torch.empty(h, device="cuda")
    dr, du = call(None, dwa, None, None)
    torch.cuda.synchronize()
    exact, bound = ref.block_norm_backward(e["u"], e["r"], e["dr_out"], e["dxn"], None, e["w_before"], e["gate"], 0.75,
                                           np.float32(eps).item(), True, bits)
    for name, got, v, b in zip(("dr", "du", "dw_after"), (dr, du, dwa), exact, bound):
        check(name, got.float().cpu().numpy(), v, b, "weight of ones")


@pytest.mark.parametrize("resid", ["float32", "bfloat16"])
@pytest.mark.parametrize("h", [64, 1024, 2048, 4096, 8192])
def test_norm_forward_in_place(h, resid):
    torch, *_ = _lib()
    from paper_2609_36301_amd import layer
    T, k = 37, 3
    dtype = getattr(torch, resid)
    gen = torch.Generator(device="cuda").manual_seed(h)
    r = torch.empty((T, h), device="cuda").normal_(generator=gen).to(dtype)
    y = torch.empty((T, k, h), device="cuda").normal_(generator=gen).bfloat16()
    w = torch.rand(h, device="cuda", generator=gen)
    announce("block_norm in place h=%d %s" % (h, resid))
    want = layer.BlockNorm(T, h, k, resid_dtype=dtype, save_u=True)(r, y, w_after=w, w_before=w)
    here = r.clone()
    got = layer.BlockNorm(T, h, k, resid_dtype=dtype, save_u=True, inplace=True)(here, y, w_after=w, w_before=w)
    assert got.r is here and torch.equal(here, want.r) and torch.equal(got.xn, want.xn) and torch.equal(got.u, want.u)


@pytest.mark.parametrize("name", ["few_rows", "ragged_dropped", "tiles_of_128_wide", "tiles_of_256", "runs_skewed"])
def test_ffn_backward_without_the_gates_gradient(name):
    torch, lib, ok, stream = _lib()
    from paper_2609_36301_amd import layer
    kw = CASES[name]
    shape = [kw[n] for n in ("T", "h", "s", "M", "k")]
    idx, bits, gate, _ = make(**kw, seed=2)
    d, i, o, s, g = on_device(idx, bits, gate, kw["M"])
    announce("more_expert_ffn_backward without dgate, %s" % name)
    want = layer.expert_ffn_backward(d["x"], d["W1t"], d["W2t"], i, o, s, g, d["du"])
    out = [torch.empty_like(t) for t in (want.dx, want.dW1t, want.dW2t)]
    ws = torch.empty(layer.expert_ffn_backward_workspace_size(*shape), dtype=torch.uint8, device="cuda")
    ok(lib.more_expert_ffn_backward(_p(d["x"]), _p(d["W1t"]), _p(d["W2t"]), *shape, _p(i), _p(o), _p(s), _p(g), _p(d["du"]),
                                    *map(_p, out), None, _p(ws), ws.numel(), stream), "more_expert_ffn_backward")
    torch.cuda.synchronize()
    for a, b in zip(out, (want.dx, want.dW1t, want.dW2t)):
        assert torch.equal(a, b)


def test_ffn_backward_of_no_tokens_without_buffers():
    torch, lib, ok, stream = _lib()
    M, h, s = 5, 48, 24
    W1, W2 = torch.ones((M, 2 * s, h), dtype=torch.bfloat16, device="cuda"), torch.ones((M, h, s), dtype=torch.bfloat16, device="cuda")
    dW1, dW2 = torch.full_like(W1, 7.0), torch.full_like(W2, 7.0)
    offsets = torch.zeros(M + 1, dtype=torch.int32, device="cuda")
    announce("more_expert_ffn_backward, no tokens, no workspace")
    ok(lib.more_expert_ffn_backward(None, _p(W1), _p(W2), 0, h, s, M, 2, None, _p(offsets), None, None, None, None, _p(dW1),
                                    _p(dW2), None, None, 0, stream), "more_expert_ffn_backward")
    torch.cuda.synchronize()
    assert not dW1.any() and not dW2.any()


def test_clip_of_no_tensors_without_the_norm_and_half_in_place():
    torch, lib, ok, stream = _lib()
    ws, norm = torch.empty(4096, dtype=torch.uint8, device="cuda"), torch.full((), 7.0, device="cuda")
    announce("more_grad_clip of no tensors, without the norm, half in place")
    ok(lib.more_grad_clip(None, None, None, None, 0, 1.0, 1e-6, _p(norm), _p(ws), ws.numel(), stream), "more_grad_clip")
    assert float(norm) == 0.0
    a, b = torch.full((100,), 3.0, device="cuda"), torch.full((77,), 4.0, device="cuda").bfloat16()
    exact = (100 * 9.0 + 77 * 16.0) ** 0.5
    for max_norm in (exact / 2, 2 * exact):  # scaling, and a factor of one
        here, out = a.clone(), torch.full_like(b, 7.0)
        ins, outs = (ctypes.c_void_p * 2)(_p(here), _p(b)), (ctypes.c_void_p * 2)(_p(here), _p(out))
        ok(lib.more_grad_clip(ins, outs, (ctypes.c_int64 * 2)(100, 77), (ctypes.c_int32 * 2)(32, 16), 2, max_norm, 1e-6, None,
                              _p(ws), ws.numel(), stream), "more_grad_clip")
        c = min(1.0, max_norm / (exact + 1e-6))
        assert bool(((here.double() / (3 * c) - 1).abs() <= 2.1 * ref.E32 + ref.E32).all())
        assert bool(((out.double() / (4 * c) - 1).abs() <= ref.E16 + 2.1 * ref.E32).all()) and bool((b == 4).all())
