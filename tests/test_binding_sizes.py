"""Sizes beyond the library's integers are refused by the binding, not cut to what is left of them (CPU: nothing is launched)."""
import os

import pytest

from paper_2609_36301_amd import _lib

torch = pytest.importorskip("torch")
WRAP = 1 << 32  # a size that is this much too large would be taken for the right one


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2609_36301_amd import build
        build.build(verbose=False)


def refused(f, *args, **kw):
    with pytest.raises(_lib.MoreError) as e:
        f(*args, **kw)
    assert e.value.status == _lib.ERR_UNSUPPORTED


def meta(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="meta")


def sizes():
    from paper_2609_36301_amd import layer, linear, router
    linear_sizes = (4, 16, 8, 2, 1)
    lowrank = (256, 512, 16, 256, 8)
    return [(linear.expert_linear_workspace_size, linear_sizes), (linear.expert_linear_backward_workspace_size, linear_sizes),
            (linear.expert_linear_q8_workspace_size, linear_sizes), (linear.expert_linear_plan, linear_sizes),
            (layer.expert_ffn_workspace_size, (4, 64, 64, 2, 1)), (layer.expert_ffn_backward_workspace_size, (4, 64, 64, 2, 1)),
            (layer.expert_ffn_plan, (4, 64, 64, 2, 1)), (layer.block_norm_backward_workspace_size, (4, 64)),
            (router.lowrank_workspace_size, lowrank), (router.lowrank_plan, lowrank), (router.lowrank_route, lowrank),
            (router.lowrank_train_workspace_size, lowrank), (router.lowrank_backward_workspace_size, lowrank),
            (router.fullrank_workspace_size, (256, 512, 256, 8)), (router.fullrank_fused_workspace_size, (256, 512, 256, 8))]


@pytest.mark.parametrize("i", range(15))
def test_queries(i):
    f, good = sizes()[i]
    f(*good)
    refused(f, (1 << 64) + good[0], *good[1:])
    for at in range(1, len(good)):  # (T has 64 bits)
        for far in (WRAP, -WRAP):
            refused(f, *good[:at], good[at] + far, *good[at + 1:])


@pytest.mark.parametrize("at", range(1, 5))
def test_linear_maps(at):
    from paper_2609_36301_amd import linear
    shape = [4, 16, 8, 2, 1]
    shape[at] += WRAP
    for call in (linear.ExpertLinear, linear.ExpertLinearBackward, linear.ExpertLinearQ8):
        refused(call, *shape, device="cuda:0")


def test_linear_maps_of_wide_tensors():
    import paper_2609_36301_amd as more
    i32 = torch.int32
    idx, offsets, srt = meta(4, 1, dtype=i32), meta(3, dtype=i32), meta(4, dtype=i32)
    refused(more.expert_linear, meta(4, WRAP + 16), meta(2, 8, WRAP + 16), idx, offsets, srt)
    refused(more.expert_linear_backward, meta(4, 16), meta(2, WRAP + 8, 16), idx, offsets, srt, meta(4, WRAP + 8))
    refused(more.expert_linear_q8, meta(4, WRAP + 16, dtype=torch.int8), meta(4), meta(2, 8, WRAP + 16, dtype=torch.int8), meta(2, 8),
            idx, offsets, srt)


@pytest.mark.parametrize("gated", [False, True])
def test_quantize_rows(gated):
    import paper_2609_36301_amd as more
    from paper_2609_36301_amd import linear
    refused(linear.QuantizeRows, 1, WRAP + 16, gated=gated, device="cuda:0")
    refused(more.quantize_rows, meta(1, (WRAP + 16) * (2 if gated else 1)), gated=gated)


def test_distillation():
    import paper_2609_36301_amd as more
    from paper_2609_36301_amd import distill
    for V, k in ((WRAP + 64, 2), (64, WRAP + 2)):
        refused(distill.Distill, 1, V, k, device="cuda:0")
        refused(distill.Distill, 1, V, k, gradient=True, inplace=True, device="cuda:0")
        refused(distill.DistillBackward, 1, V, k, device="cuda:0")
        ids, values, row = meta(1, k, dtype=torch.int32), meta(1, k, dtype=torch.float32), meta(1, dtype=torch.float32)
        refused(more.distill_loss, meta(1, V), ids, values)
        refused(more.distill_backward, meta(1, V), row, row, ids, values, row)


def test_sort_histogram_and_norm():
    from paper_2609_36301_amd import layer, router
    refused(router.DispatchSorter, 4, 2, WRAP + 8)
    refused(router.DispatchSorter, 4, WRAP + 2, 8)
    for shape in ((4, WRAP + 64, 1), (4, 64, WRAP + 1)):
        refused(layer.BlockNorm, *shape, device="cuda:0")
