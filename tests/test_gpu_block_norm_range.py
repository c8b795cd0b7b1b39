"""The norms' backward pass where the factor of a row is far from one: rows of zeros with a small eps (1 / rms is
then 1 / sqrt(eps)) and rows whose root mean square is large (marked `gpu`).  The bounds are those of layer_ref.py."""
import numpy as np
import pytest

import layer_ref as ref
from gpu_util import announce, require_gpu, to_dev
from test_gpu_block_norm import _case, _dev, _f64, _resid
from test_gpu_ffn import check

pytestmark = pytest.mark.gpu

NAMES = ("dr", "du", "dw_after", "dw_before", "dgate")


def _backward(a, block, alpha, eps, bits):
    torch = require_gpu()
    from paper_2609_36301_amd import layer
    a = {n: v if block or n in ("r", "dxn", "w_before") else None for n, v in a.items()}
    d, e = _dev(a), {n: _f64(v) for n, v in a.items()}
    out = layer.block_norm_backward(d["u"], d["r"], None, d["dxn"], w_after=d["w_after"], w_before=d["w_before"],
                                    gate=d["gate"], alpha=alpha, eps=eps)
    torch.cuda.synchronize()
    want, bound = ref.block_norm_backward(e["u"], e["r"], None, e["dxn"], e["w_after"], e["w_before"], e["gate"], alpha,
                                          np.float32(eps).item(), True, bits)
    for name, v, b in zip(NAMES, want, bound):
        assert (getattr(out, name) is None) == (v is None), name
        if v is not None:
            check(name, getattr(out, name).float().cpu().numpy(), v, b, "eps %g" % eps)


@pytest.mark.parametrize("block", [True, False], ids=["block", "norm_alone"])
@pytest.mark.parametrize("h,bits", [(64, 32), (1040, 16), (4112, 32)])
@pytest.mark.parametrize("eps", [1e-12, 1e-27, 1e-36])
def test_rows_of_zeros_with_a_small_eps(eps, h, bits, block):
    a = _case(9, h, 1, bits, True, seed=7)
    a["r"][3:5] = 0
    a["u"][4:6] = 0
    announce("block_norm_backward, zero rows, eps=%g h=%d resid=%d block=%s" % (eps, h, bits, block))
    _backward(a, block, 0.75, eps, bits)


@pytest.mark.parametrize("block", [True, False], ids=["block", "norm_alone"])
@pytest.mark.parametrize("h,bits", [(64, 32), (1040, 16), (4112, 32)])
@pytest.mark.parametrize("rms", [2.0 ** 30, 2.0 ** 44, 2.0 ** 52])
def test_rows_of_large_values(rms, h, bits, block):
    a = _case(9, h, 1, bits, True, seed=8, zero_rows=False)
    rng = np.random.default_rng(9)
    a["r"] = _resid(rng.standard_normal((9, h)) * rms, bits)
    a["u"] = ref.to_bf16(rng.standard_normal((9, h)) * rms)
    # gradients of a size that the results keep: those of r are 1 / rms of those of xn, those of u 1 / rms of r's
    a["dxn"] = ref.to_bf16(rng.standard_normal((9, h)) * rms)
    announce("block_norm_backward, rows of about %g, h=%d resid=%d block=%s" % (rms, h, bits, block))
    _backward(a, block, 0.75, 1e-6, bits)
