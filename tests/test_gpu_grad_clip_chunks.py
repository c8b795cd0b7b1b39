"""Clipping with work items of every length: 2048 elements for small sets, and up to 16384 for sets of more than
2^22 elements, with tensors that end one element before, at and behind an item's end (marked `gpu`).  The
tolerances are those of test_gpu_grad_clip.py."""
import pytest

from gpu_util import announce, require_gpu
from test_gpu_grad_clip import _check, _grads

pytestmark = pytest.mark.gpu


def _edges(chunk, total):
    """Tensors around multiples of `chunk`, filled up to `total` elements by two large ones of either type."""
    edges = [(n, bits) for bits in (32, 16) for n in (1, chunk - 1, chunk, chunk + 1, 3 * chunk - 5, 3 * chunk + 11)]
    rest = total - sum(n for n, _ in edges)
    return edges + [(rest // 2, 16), (rest - rest // 2, 32)]


SETS = {"2048": [e for e in _edges(2048, 60000)], "4096": _edges(4096, (2 << 22) + 77),
        "6144": _edges(6144, (3 << 22) + 5), "16384": _edges(16384, (8 << 22) + 3)}


@pytest.mark.parametrize("name", list(SETS))
@pytest.mark.parametrize("aligned", [True, False], ids=["aligned", "odd_start"])
def test_clip(name, aligned):
    torch = require_gpu()
    from paper_2609_36301_amd import layer
    sizes = SETS[name]
    announce("clip items of %s elements, %d tensors, aligned=%s" % (name, len(sizes), aligned))
    before = _grads(torch, [(n + (not aligned), bits) for n, bits in sizes], seed=3)
    before = [g if aligned else g[1:] for g in before]
    out = [torch.full_like(g, 7.0) for g in before]
    norm, got = layer.GradClipper(before, 0.25, out=out)()
    _check(torch, before, got, norm, 0.25)
    # in place, on views with a guard element on either side
    held = [torch.full((g.numel() + 2 + 2 * aligned * (8 if g.dtype == torch.bfloat16 else 4),), 5.0, dtype=g.dtype,
                       device="cuda") for g in before]
    start = [1 if not aligned else 8 if g.dtype == torch.bfloat16 else 4 for g in before]
    views = [t[a:a + g.numel()] for t, a, g in zip(held, start, before)]
    for v, g in zip(views, before):
        v.copy_(g)
    norm = layer.clip_gradients(views, 0.25)
    _check(torch, before, views, norm, 0.25)
    for t, a, g in zip(held, start, before):
        assert bool((t[:a] == 5).all()) and bool((t[a + g.numel():] == 5).all())
