"""Every form of the experts' kernels on values: tiles of every size, the decode kernels (32 rows) with either ring,
spans of several column steps with a ragged last one, contractions of several stages, weight-gradient tiles of both
sizes, one and two addends.  Each case names the form that it is there for, and the plan of the shape has to be that
form, so that a later rule cannot take a case elsewhere unnoticed (values marked `gpu`; the plans are host queries)."""
import numpy as np
import pytest

import layer_ref as ref
from gpu_util import announce, require_gpu
from test_gpu_ffn import check, make, on_device

# name: (shape, the forward plan, the backward plan), as far as the case is about them
FORMS = {
    "decode_ring_of_two": (dict(T=700, h=4112, s=72, M=140, k=4, drop=0.05),
                           dict(tile_rows=32, addends=1, span=512, stages=2), dict(tile_rows=32, addends=1, span=512)),
    "decode_ring_of_three": (dict(T=4336, h=704, s=80, M=396, k=1, drop=0.02),
                             dict(tile_rows=32, addends=1, span=512, stages=3),
                             dict(tile_rows=32, addends=1, span=512, dw_tile=128, dw1_span=512, dw2_span=512)),
    "decode_short_spans": (dict(T=500, h=1040, s=40, M=150, k=3, drop=0.1),
                           dict(tile_rows=32, addends=1, span=128, stages=3), dict(tile_rows=32, addends=1, span=128)),
    "decode_ring_of_two_two_addends": (dict(T=1024, h=2064, s=32, M=900, k=1, drop=0.1),
                                       dict(tile_rows=32, addends=2, span=512, stages=2),
                                       dict(tile_rows=32, addends=2, span=512, dw1_span=512, dw2_span=512)),
    "decode_ring_of_three_two_addends": (dict(T=330, h=2064, s=24, M=200, k=4, drop=0.1),
                                         dict(tile_rows=32, addends=2, span=512, stages=3),
                                         dict(tile_rows=32, addends=2, span=512)),
    "decode_past_2_16_experts": (dict(T=5000, h=32, s=40, M=70000, k=1, drop=0.05, repeat=True),
                                 dict(tile_rows=32, addends=1, stages=2), dict(tile_rows=32, dw1_span=512)),
    "tiles_of_64_long_spans": (dict(T=10540, h=672, s=72, M=387, k=1, drop=0.01),
                               dict(tile_rows=64, addends=1, span=512, stages=3),
                               dict(tile_rows=64, span=512, dw_tile=128, dw1_span=512, dw2_span=512)),
    "tiles_of_64_hot": (dict(T=900, h=144, s=136, M=16, k=3, hot=0.6, drop=0.03),
                        dict(tile_rows=64, span=128, stages=3), dict(tile_rows=64, span=128)),
    "tiles_of_128_long_spans": (dict(T=28282, h=624, s=72, M=444, k=1, drop=0.01),
                                dict(tile_rows=128, addends=1, span=512, stages=2),
                                dict(tile_rows=128, span=512, dw_tile=128, dw1_span=512, dw2_span=512)),
    "tiles_of_256_long_spans": (dict(T=31185, h=1168, s=80, M=227, k=1, drop=0.01),
                                dict(tile_rows=256, addends=1, span=512, stages=2),
                                dict(tile_rows=256, span=512, dw1_span=512, dw2_span=512)),
    "tiles_of_256_and_runs": (dict(T=15410, h=400, s=288, M=4, k=1, hot=0.2, drop=0.01),
                              dict(tile_rows=128), dict(tile_rows=256, dw_tile=128, dw_runs=4)),
    "large_weight_gradient_tiles_few_rows": (dict(T=218, h=656, s=264, M=290, k=1),
                                             dict(tile_rows=32, addends=1, stages=3),
                                             dict(tile_rows=32, dw_tile=256, dw1_span=512, dw2_span=512)),
    "no_tiles_shared_columns": (dict(T=3, h=528, s=264, M=9, k=2, drop=0.2), dict(tile_rows=0, addends=2, span=32),
                                dict(tile_rows=32, addends=2)),
    "no_tiles": (dict(T=60, h=1040, s=40, M=300, k=4, drop=0.1), dict(tile_rows=0, addends=2, span=256),
                 dict(tile_rows=32, addends=2)),
}


@pytest.mark.parametrize("name", list(FORMS))
def test_plan(name):
    from paper_2609_36301_amd import expert_ffn_plan
    kw, *plans = FORMS[name]
    for backward, want in enumerate(plans):
        plan = expert_ffn_plan(kw["T"], kw["h"], kw["s"], kw["M"], kw["k"], backward=bool(backward))
        assert {field: plan[field] for field in want} == want, ("backward" if backward else "forward", plan)


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(FORMS))
def test_values(name):
    kw, forward, backward = FORMS[name]
    M = kw["M"]
    idx, bits, gate, exact = make(**kw, seed=11)
    torch = require_gpu()
    from paper_2609_36301_amd import layer
    announce("expert_ffn and its backward pass, %s %s" % (name, kw))
    d, i, o, s, g = on_device(idx, bits, gate, M)
    y = layer.expert_ffn(d["x"], d["W1t"], d["W2t"], i, o, s, g)
    got = layer.expert_ffn_backward(d["x"], d["W1t"], d["W2t"], i, o, s, g, d["du"])
    torch.cuda.synchronize()
    given = (exact["x"], exact["W1t"], exact["W2t"], idx, exact["gate"])
    want, bound = ref.ffn(*given, planes=forward.get("addends", 1))
    check("y", y.float().cpu().numpy(), want, bound, name)
    assert np.all(y.float().cpu().numpy()[(idx.ravel() < 0) | (idx.ravel() >= M)] == 0)
    want, bound = ref.ffn_backward(*given, exact["du"], planes=backward.get("addends", 1))
    for field, v, b in zip(("dx", "dW1t", "dW2t", "dgate"), want, bound):
        check(field, getattr(got, field).float().cpu().numpy(), v, b, name)


def test_plan_refuses():
    import ctypes
    from paper_2609_36301_amd import _lib
    lib, plan = _lib.load(), _lib.ExpertPlan()
    for args, status in (((64, 64, 16, 8, 2), _lib.OK), ((0, 64, 16, 8, 2), _lib.OK), ((-1, 64, 16, 8, 2), _lib.ERR_INVALID_ARG),
                         ((64, 72, 16, 8, 2), _lib.ERR_UNSUPPORTED), ((64, 64, 16, 8, 33), _lib.ERR_UNSUPPORTED)):
        for backward in (0, 1):
            assert lib.more_expert_ffn_plan(*args, 0, backward, ctypes.byref(plan)) == status
    assert lib.more_expert_ffn_plan(64, 64, 16, 8, 2, 0, 0, None) == _lib.ERR_INVALID_ARG
