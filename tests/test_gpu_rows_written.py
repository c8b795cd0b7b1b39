"""Distillation and quantised rows into outputs full of NaN (of sevens, in 8 bits), in every form: what a call leaves unwritten
is seen."""
import numpy as np
import pytest

import linear_ref as ref
from gpu_util import announce, require_gpu, to_dev
from layer_ref import from_bf16, to_bf16
from test_gpu_distill import LENGTHS, case, close, rows_on_device

pytestmark = pytest.mark.gpu

NAN = float("nan")


@pytest.mark.parametrize("bits", [16, 32])
@pytest.mark.parametrize("V", LENGTHS + [200001])
def test_distillation(V, bits):
    torch = require_gpu()
    from paper_2609_36301_amd import distill
    T, tau, dtype = 6, 2.0, torch.float32 if bits == 32 else torch.bfloat16
    for k in (4, 70):
        z, ids, values, w = case(V + k, T, V, k, bits)
        ld = V + 5
        announce("distill over NaN V=%d k=%d bits=%d" % (V, k, bits))
        (loss, m, Z, grad), (bl, bZ, bg) = ref.distill(z, ids, values.astype(np.float64), tau, w.astype(np.float64), bits)
        logits = rows_on_device(z, bits, ld, 1)[1]
        args = [to_dev(v) for v in (ids, values, w)]
        options = dict(dtype=dtype, temperature=tau, ld=ld)
        both, alone = distill.Distill(T, V, k, gradient=True, **options), distill.Distill(T, V, k, **options)
        back = distill.DistillBackward(T, V, k, **options)
        for t in (both.loss, both.m, both.Z, both.dlogits, alone.loss, alone.m, alone.Z, back.dlogits):
            t.fill_(NAN)
        both(logits, *args)
        alone(logits, *args[:2])
        back(logits, alone.m, alone.Z, *args)
        for d in (both, alone):
            close(d.loss, loss, bl, "loss")
            close(d.Z, Z, bZ, "Z")
            assert np.array_equal(d.m.cpu().numpy().astype(np.float64), m)
        for g in (both.dlogits, back.dlogits):
            close(g, grad, bg, "dlogits")


@pytest.mark.parametrize("width", [16, 512, 528, 1024, 1040, 2048, 2064, 8192, 8208, 32768, 32784, 65536])
def test_quantised_rows(width):
    require_gpu()
    from paper_2609_36301_amd import linear
    rng = np.random.default_rng(width)
    x = to_bf16(rng.standard_normal((9, width)))
    x[4] = 0
    announce("quantize_rows over sevens width=%d" % width)
    call = linear.QuantizeRows(9, width)
    call.q.fill_(7)
    call.scale.fill_(NAN)
    got = call(to_dev(x))
    q, scale = ref.quantize(from_bf16(x))
    assert np.array_equal(got.q.cpu().numpy(), q) and np.array_equal(got.scale.cpu().numpy(), scale)
