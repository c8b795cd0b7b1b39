"""The norms at a block's ends and their backward pass against the 64-bit reference, within the bounds of
layer_ref.py (marked `gpu`)."""
import numpy as np
import pytest

import layer_ref as ref
from gpu_util import announce, require_gpu, to_dev
from test_gpu_ffn import check

pytestmark = pytest.mark.gpu

# every row layout (one, four or eight waves, one or two chunks per lane) with full and ragged widths
WIDTHS = [16, 512, 528, 1024, 1040, 2048, 2064, 4096, 4112, 8192]


def _resid(a, bits):
    return ref.to_bf16(a) if bits == 16 else a.astype(np.float32)


def _f64(a):
    return None if a is None else ref.from_bf16(a) if a.dtype == np.uint16 else a.astype(np.float64)


def _case(T, h, k, bits, gated, seed=0, zero_rows=True):
    rng = np.random.default_rng(seed + T + h + k)
    a = {"r": _resid(rng.standard_normal((T, h)) * 2, bits), "y": ref.to_bf16(rng.standard_normal((T, max(k, 1), h)) * 0.4),
         "w_after": (1 + 0.1 * rng.standard_normal(h)).astype(np.float32),
         "w_before": (1 + 0.1 * rng.standard_normal(h)).astype(np.float32),
         "gate": rng.random(T).astype(np.float32) if gated else None,
         "u": ref.to_bf16(rng.standard_normal((T, h))), "dr_out": _resid(rng.standard_normal((T, h)), bits),
         "dxn": ref.to_bf16(rng.standard_normal((T, h))), "dxn32": rng.standard_normal((T, h)).astype(np.float32)}
    if zero_rows and T > 2:  # a token without a block output (all entries dropped), and an empty residual
        a["y"][1] = a["u"][1] = 0
        a["r"][2] = 0
    return a


def _dev(a):
    return {n: None if v is None else to_dev(v) for n, v in a.items()}


FORWARD = ([(5, h, 2, 16, True, True) for h in WIDTHS] + [(3, h, 1, 32, False, False) for h in WIDTHS[::2]] +
           [(1, 4096, 16, 16, False, True), (1, 64, 32, 32, True, True), (130, 272, 5, 32, True, True),
            (1000, 96, 3, 16, True, False), (67, 2032, 8, 32, False, True)])


@pytest.mark.parametrize("T,h,k,bits,gated,after", FORWARD, ids=lambda v: str(v))
def test_forward(T, h, k, bits, gated, after):
    torch = require_gpu()
    from paper_2609_36301_amd import layer
    a = _case(T, h, k, bits, gated)
    d = _dev(a)
    announce("block_norm T=%d h=%d k=%d resid=%d gated=%s after=%s" % (T, h, k, bits, gated, after))
    out = layer.block_norm(d["r"], d["y"], w_after=d["w_after"], w_before=d["w_before"], gate=d["gate"], norm_after=after,
                           alpha=0.75, eps=1e-5, save_u=True)
    torch.cuda.synchronize()
    e = {n: _f64(v) for n, v in a.items()}
    want, bound = ref.block_norm(e["r"], e["y"], e["w_after"], e["w_before"], e["gate"], 0.75, np.float32(1e-5).item(),
                                 after, bits)
    for name, v, b in zip(("r", "xn", "u"), want, bound):
        check(name, getattr(out, name).float().cpu().numpy(), v, b, "block_norm")


def test_forms():
    """Only the norm; no norm after the block's end; no weight; in place."""
    torch = require_gpu()
    from paper_2609_36301_amd import layer
    T, h, k = 33, 320, 3
    a = _case(T, h, k, 16, False)
    d, e = _dev(a), {n: _f64(v) for n, v in a.items()}
    announce("block_norm forms T=%d h=%d" % (T, h))
    eps = np.float32(1e-6).item()
    first = layer.block_norm(d["r"], w_before=d["w_before"])
    assert first.r is d["r"] and first.u is None
    want, bound = ref.block_norm(e["r"], None, None, e["w_before"], None, 1.0, eps, True, 16)
    check("xn", first.xn.float().cpu().numpy(), want[1], bound[1], "norm only")
    last = layer.block_norm(d["r"], d["y"].view(T * k, h), alpha=0.5)
    assert last.xn is None
    want, bound = ref.block_norm(e["r"], e["y"], None, None, None, 0.5, eps, True, 16)
    check("r", last.r.float().cpu().numpy(), want[0], bound[0], "last")
    here = layer.BlockNorm(T, h, k, alpha=0.5, inplace=True)
    r = d["r"].clone()
    out = here(r, d["y"])
    assert out.r is r and torch.equal(r, last.r)
    torch.cuda.synchronize()


BACKWARD = ([(7, h, 16, True, True, "both") for h in WIDTHS] + [(3, h, 32, False, True, "bf16") for h in WIDTHS[1::2]] +
            [(1, 1024, 32, True, True, "fp32"), (5000, 48, 32, True, True, "both"), (1500, 2032, 16, False, False, "bf16"),
             (4099, 528, 32, True, False, "fp32"), (9, 64, 32, True, True, "none")])


@pytest.mark.parametrize("T,h,bits,gated,after,grads", BACKWARD, ids=lambda v: str(v))
def test_backward(T, h, bits, gated, after, grads):
    torch = require_gpu()
    from paper_2609_36301_amd import layer
    a = _case(T, h, 1, bits, gated, seed=5)
    if grads in ("fp32", "none"):
        a["dxn"] = None
    if grads in ("bf16", "none"):
        a["dxn32"] = None
    if grads == "none":
        a["w_before"] = None
    if grads == "fp32":
        a["dr_out"] = None
    d, e = _dev(a), {n: _f64(v) for n, v in a.items()}
    announce("block_norm_backward T=%d h=%d resid=%d gated=%s after=%s grads=%s" % (T, h, bits, gated, after, grads))
    out = layer.block_norm_backward(d["u"], d["r"], d["dr_out"], d["dxn"], dxn32=d["dxn32"], w_after=d["w_after"],
                                    w_before=d["w_before"], gate=d["gate"], norm_after=after, alpha=0.75, eps=1e-3)
    torch.cuda.synchronize()
    dxn = None if grads == "none" else sum(v for v in (e["dxn"], e["dxn32"]) if v is not None)
    want, bound = ref.block_norm_backward(e["u"], e["r"], e["dr_out"], dxn, e["w_after"], e["w_before"], e["gate"], 0.75,
                                          np.float32(1e-3).item(), after, bits)
    for name, v, b in zip(("dr", "du", "dw_after", "dw_before", "dgate"), want, bound):
        got = getattr(out, name)
        assert (got is None) == (v is None), name
        if got is not None:
            check(name, got.float().cpu().numpy(), v, b, "block_norm_backward")


@pytest.mark.parametrize("T,h", [(40, 2064), (40, 128)])
def test_backward_of_the_norm_alone_and_no_tokens(T, h):
    torch = require_gpu()
    from paper_2609_36301_amd import layer
    a = _case(T, h, 1, 32, False)
    d, e = _dev(a), {n: _f64(v) for n, v in a.items()}
    announce("block_norm_backward without a block T=%d h=%d" % (T, h))
    out = layer.block_norm_backward(None, d["r"], d["dr_out"], d["dxn"], w_before=d["w_before"], eps=1e-3)
    torch.cuda.synchronize()
    want, bound = ref.block_norm_backward(None, e["r"], e["dr_out"], e["dxn"], None, e["w_before"], None, 1.0,
                                          np.float32(1e-3).item(), True, 32)
    assert out.du is None and out.dw_after is None and out.dgate is None
    check("dr", out.dr.cpu().numpy(), want[0], bound[0], "norm alone")
    check("dw_before", out.dw_before.cpu().numpy(), want[3], bound[3], "norm alone")
    empty = torch.empty((0, h), device="cuda")
    e16 = empty.bfloat16()
    out = layer.block_norm_backward(e16, empty, empty, e16, w_after=d["w_after"], w_before=d["w_before"])
    assert not out.dw_after.any() and not out.dw_before.any()
    assert layer.block_norm(empty, w_before=d["w_before"]).xn.shape == (0, h)


def test_more_rows_than_a_launch_takes():
    """2^26 rows of 16 columns and a few more: the last rows, and those at the seam."""
    torch = require_gpu()
    from paper_2609_36301_amd import layer
    T, h = (1 << 26) + 5, 16
    announce("block_norm T=%d h=%d" % (T, h))
    r = torch.empty((T, h), dtype=torch.bfloat16, device="cuda").normal_()
    y = torch.empty((T, h), dtype=torch.bfloat16, device="cuda").normal_()
    gate = torch.rand(T, device="cuda")
    w = torch.rand(h, device="cuda") + 0.5
    out = layer.block_norm(r, y, w_after=w, w_before=w, gate=gate, save_u=True)
    for rows in (slice(0, 3), slice((1 << 24) - 2, (1 << 24) + 2), slice((1 << 25) - 1, (1 << 25) + 1), slice(T - 7, T)):
        e = lambda t: t[rows].double().cpu().numpy()  # noqa: E731
        wd = w.double().cpu().numpy()
        want, bound = ref.block_norm(e(r), e(y)[:, None], wd, wd, e(gate), 1.0, np.float32(1e-6).item(), True, 16)
        for name, v, b in zip(("r", "xn", "u"), want, bound):
            check(name, getattr(out, name)[rows].float().cpu().numpy(), v, b, str(rows))


def test_binding_refuses():
    torch = require_gpu()
    from paper_2609_36301_amd import layer
    r = torch.zeros((4, 64), device="cuda")
    w = torch.ones(64, device="cuda")
    call = layer.BlockNorm(4, 64, 2, resid_dtype=torch.float32)
    with pytest.raises(ValueError, match="y must be given"):
        call(r, w_before=w)
    with pytest.raises(TypeError, match="r must be torch.float32"):
        call(r.bfloat16(), torch.zeros((8, 64), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError, match="y must be a contiguous"):
        call(r, torch.zeros((4, 3, 64), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(TypeError, match="w_before"):
        call(r, torch.zeros((8, 64), dtype=torch.bfloat16, device="cuda"), w_before=w.bfloat16())
    with pytest.raises(ValueError, match="gate must be given"):
        layer.BlockNormBackward(4, 64, resid_dtype=torch.float32, gated=True)(None, r, r)
    with pytest.raises(layer._lib.MoreError):
        layer.block_norm(r, w_before=w, eps=0.0)
