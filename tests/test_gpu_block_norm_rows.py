"""The norms' backward pass where a workgroup takes several rows one after the other (more than 1024 of them, or 4096
on rows of one wave), on every row layout: one, four and eight waves, one and two chunks per lane; with a block and
for the norm alone.  And the forward pass of the norm alone on every layout (marked `gpu`)."""
import numpy as np
import pytest

import layer_ref as ref
from gpu_util import announce, require_gpu
from test_gpu_block_norm import WIDTHS, _case, _dev, _f64
from test_gpu_ffn import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("block", [True, False], ids=["block", "norm_alone"])
@pytest.mark.parametrize("T,h,bits", [(8200, 272, 16), (4500, 1024, 32), (2100, 2032, 32), (3100, 2048, 16), (2100, 2064, 16),
                                      (2100, 4096, 32), (2100, 4112, 16), (1300, 8192, 16)])
def test_backward_of_several_rows_per_workgroup(T, h, bits, block):
    torch = require_gpu()
    from paper_2609_36301_amd import layer
    a = _case(T, h, 1, bits, True, seed=12)
    if not block:
        a["u"] = a["w_after"] = a["gate"] = None
    d, e = _dev(a), {n: _f64(v) for n, v in a.items()}
    announce("block_norm_backward T=%d h=%d resid=%d block=%s" % (T, h, bits, block))
    out = layer.block_norm_backward(d["u"], d["r"], d["dr_out"], d["dxn"], dxn32=d["dxn32"], w_after=d["w_after"],
                                    w_before=d["w_before"], gate=d["gate"], alpha=0.75, eps=1e-3)
    torch.cuda.synchronize()
    want, bound = ref.block_norm_backward(e["u"], e["r"], e["dr_out"], e["dxn"] + e["dxn32"], e["w_after"], e["w_before"],
                                          e["gate"], 0.75, np.float32(1e-3).item(), True, bits)
    for name, v, b in zip(("dr", "du", "dw_after", "dw_before", "dgate"), want, bound):
        got = getattr(out, name)
        assert (got is None) == (v is None), name
        if got is not None:
            check(name, got.float().cpu().numpy(), v, b, "block_norm_backward")


@pytest.mark.parametrize("bits", [16, 32])
@pytest.mark.parametrize("h", WIDTHS)
def test_forward_of_the_norm_alone(h, bits):
    torch = require_gpu()
    from paper_2609_36301_amd import layer
    a = _case(11, h, 0, bits, False, seed=13)
    d, e = _dev(a), {n: _f64(v) for n, v in a.items()}
    announce("block_norm without a block h=%d resid=%d" % (h, bits))
    out = layer.block_norm(d["r"], w_before=d["w_before"], eps=1e-6)
    torch.cuda.synchronize()
    want, bound = ref.block_norm(e["r"], None, None, e["w_before"], None, 1.0, np.float32(1e-6).item(), True, bits)
    check("xn", out.xn.float().cpu().numpy(), want[1], bound[1], "norm alone")
