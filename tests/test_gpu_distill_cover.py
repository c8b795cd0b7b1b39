"""Distillation where a teacher's entries cover most classes, or all: loss and gradient at every temperature against 60
digits, with bounds relative to them."""
import numpy as np
import pytest

import distill_ref as ref
from gpu_util import announce, require_gpu, to_dev
from layer_ref import from_bf16, to_bf16
from test_gpu_distill import close, rows_on_device

pytestmark = pytest.mark.gpu

TAUS = [2.0 ** -40, 0.25, 1.0, 20.0, 256.0, 4096.0, 2.0 ** 20, 2.0 ** 40]


def case(seed, V, k, bits, repeats=False):
    """Rows that differ: all classes (as far as k goes), a teacher who leaves some out, a student who does, a teacher who says
    what the student says, a wide spread, none."""
    rng = np.random.default_rng(seed)
    T = 6
    z = rng.standard_normal((T, V))
    z[4] *= 200.0
    z = z.astype(np.float32).astype(np.float64) if bits == 32 else from_bf16(to_bf16(z))
    if repeats or k > V:
        ids = rng.integers(0, V, (T, k))
    else:
        ids = np.stack([rng.permutation(V)[:k] for _ in range(T)])
    ids = ids.astype(np.int32)
    values = rng.standard_normal((T, k)).astype(np.float32)
    ids[1, : k // 3], values[1, k // 3: k // 2] = V, -np.inf
    out = rng.random(V) < 0.3
    out[ids[2, -1]] = False
    z[2, out] = -np.inf
    ids[2, out[ids[2]]] = -1
    values[3] = z[3, ids[3]] + 3
    values[4] *= 100
    ids[5] = -1
    return z, ids, values, rng.standard_normal(T).astype(np.float32)


SHAPES = [(1, 1), (1, 3), (2, 1), (7, 7), (33, 17), (64, 64), (65, 64), (100, 64), (200, 256), (512, 300), (513, 512), (1024, 1024),
          (1500, 800), (2048, 1024)]


# (rows of a thousand classes take a second or two to 60 digits: three temperatures of them)
@pytest.mark.parametrize("bits", [16, 32])
@pytest.mark.parametrize("V,k,tau", [(V, k, tau) for V, k in SHAPES for tau in (TAUS if V < 600 else TAUS[1::3])])
def test_covered(V, k, tau, bits):
    torch = require_gpu()
    from paper_2609_36301_amd import distill_backward, distill_loss
    for repeats in (False, True) if V < 300 else (V % 2 == 1,):
        z, ids, values, w = case(V + k, V, k, bits, repeats)
        announce("distill V=%d k=%d tau=%g bits=%d repeats=%s" % (V, k, tau, bits, repeats))
        (loss, grad), (bl, bg) = ref.distill(z, ids, values.astype(np.float64), tau, w.astype(np.float64), bits)
        logits = rows_on_device(z, bits, V + 1, 1)[1]
        args = to_dev(ids), to_dev(values)
        alone = distill_loss(logits, *args, temperature=tau)
        d = distill_loss(logits, *args, to_dev(w), temperature=tau, gradient=True)
        close(d.loss, loss, bl, "loss")
        close(d.dlogits, grad, bg, "dlogits")
        assert torch.equal(alone.loss, d.loss) and torch.equal(alone.Z, d.Z) and torch.equal(alone.m, d.m)
        two = distill_backward(logits, alone.m, alone.Z, *args, to_dev(w), temperature=tau)
        assert torch.equal(two, d.dlogits)
        assert d.loss[5] == 0 and not d.dlogits[5].any()


@pytest.mark.parametrize("bits", [16, 32])
@pytest.mark.parametrize("V,k,ld,start", [(9, 9, 9, 0), (64, 40, 67, 3), (300, 200, 301, 1), (700, 512, 704, 5), (2047, 1024, 2048, 1)])
def test_covered_in_place_and_nothing_beside_the_rows(V, k, ld, start, bits):
    torch = require_gpu()
    from paper_2609_36301_amd import distill
    z, ids, values, w = case(V, V, k, bits, repeats=True)
    T, tau = len(z), 300.0
    announce("distill in place V=%d k=%d bits=%d ld=%d start=%d" % (V, k, bits, ld, start))
    dtype = torch.float32 if bits == 32 else torch.bfloat16
    args = to_dev(ids), to_dev(values)
    make = lambda **kw: distill.Distill(T, V, k, dtype=dtype, temperature=tau, ld=ld, gradient=True, **kw)  # noqa: E731
    want = make()(rows_on_device(z, bits, ld, start)[1], *args, to_dev(w))
    for backward in (False, True):
        big, logits = rows_on_device(z, bits, ld, start)
        if backward:
            back = distill.DistillBackward(T, V, k, dtype=dtype, temperature=tau, ld=ld, inplace=True)
            got = back(logits, want.m, want.Z, *args, to_dev(w))
        else:
            got = make(inplace=True)(logits, *args, to_dev(w)).dlogits
        assert got.data_ptr() == logits.data_ptr() and torch.equal(got, want.dlogits)
        beside = torch.ones_like(big, dtype=torch.bool)
        beside[start:start + T * ld].view(T, ld)[:, :V] = False
        assert (big[beside] == 7).all()


@pytest.mark.parametrize("V,k", [(40, 40), (700, 600)])
def test_covered_rows_that_have_no_loss_are_alone(V, k):
    torch = require_gpu()
    from paper_2609_36301_amd import distill_loss
    z, ids, values, w = case(V, V, k, 32)
    plain, kept = z.copy(), values.copy()
    z[1, V // 3], z[3, V // 2], z[4] = np.nan, np.inf, -np.inf
    values[2, -1] = np.nan
    announce("distill with rows of NaN V=%d k=%d" % (V, k))
    (loss, grad), (bl, bg) = ref.distill(plain, ids, kept.astype(np.float64), 50.0, w.astype(np.float64))
    d = distill_loss(rows_on_device(z, 32)[1], to_dev(ids), to_dev(values), to_dev(w), temperature=50.0, gradient=True)
    assert torch.isnan(d.loss[1:5]).all()
    good = [0, 5]
    close(d.loss[good], loss[good], bl[good], "loss")
    close(d.dlogits[good], grad[good], bg[good], "dlogits")


def test_covered_without_probability():
    """A class that the student rules out and the teacher does not: an infinite loss and the gradient of the teacher's
    share; one that neither has: nothing."""
    require_gpu()
    import torch
    from paper_2609_36301_amd import distill_loss
    announce("distill, a class that the student rules out")
    z = torch.zeros((2, 4), device="cuda")
    z[:, 1] = -float("inf")
    ids = torch.arange(4, dtype=torch.int32, device="cuda").repeat(2, 1)
    values = torch.zeros((2, 4), device="cuda")
    values[1, 1] = -1e6
    d = distill_loss(z, ids, values, temperature=2.0, gradient=True)
    assert d.loss[0] == float("inf") and d.loss[1] == 0
    # (P is 1/3, Q 1/4: five roundings each)
    want = torch.tensor([2 / 12, -2 / 4, 2 / 12, 2 / 12])
    assert (d.dlogits[0].cpu() - want).abs().max() < 10 * 2.0 ** -24 and not d.dlogits[1].any()


def test_covered_many_rows():
    """More rows than workgroups."""
    torch = require_gpu()
    from paper_2609_36301_amd import distill_loss
    for T, V, k in (((1 << 22) + 5, 2, 2), ((1 << 20) + 3, 600, 300)):
        announce("distill T=%d V=%d k=%d" % (T, V, k))
        gen = torch.Generator(device="cuda").manual_seed(3)
        z = torch.randn((1, V), device="cuda", generator=gen)
        ids = torch.randperm(V, device="cuda", generator=gen)[None, :k].int()
        values = torch.randn((1, k), device="cuda", generator=gen)
        one = distill_loss(z, ids, values, temperature=9.0, gradient=True)
        d = distill_loss(z.repeat(T, 1), ids.repeat(T, 1), values.repeat(T, 1), temperature=9.0, gradient=True)
        assert (d.loss == one.loss).all() and (d.Z == one.Z).all()
        for a in range(0, T, 1 << 18):
            assert (d.dlogits[a:a + (1 << 18)] == one.dlogits).all()
        del d


def test_covered_in_a_graph():
    torch = require_gpu()
    from paper_2609_36301_amd import distill
    z, ids, values, w = case(11, 90, 64, 32)
    announce("distill in a graph, V=90 k=64")
    logits, args = rows_on_device(z, 32)[1], [to_dev(v) for v in (ids, values, w)]
    call = distill.Distill(len(z), 90, 64, dtype=torch.float32, temperature=700.0, gradient=True)
    eager = call(logits, *args)
    want = [t.clone() for t in (eager.loss, eager.m, eager.Z, eager.dlogits)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        d = call(logits, *args)
    for _ in range(3):
        for t in (d.loss, d.m, d.Z, d.dlogits):
            t.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((d.loss, d.m, d.Z, d.dlogits), want))


@pytest.mark.parametrize("V,k", [(90, 64), (900, 512)])
def test_covered_each_output_alone(V, k):
    """The library's call with any of its outputs left out, and gradients that lie otherwise than the logits."""
    torch = require_gpu()
    from paper_2609_36301_amd import _lib, distill_loss
    z, ids, values, w = case(V, V, k, 32, repeats=True)
    T, tau = len(z), 30.0
    announce("distill V=%d k=%d, each output alone" % (V, k))
    logits, ids, values, w = rows_on_device(z, 32, V + 2, 3)[1], to_dev(ids), to_dev(values), to_dev(w)
    want = distill_loss(logits, ids, values, w, temperature=tau, gradient=True)
    stream = torch.cuda.current_stream().cuda_stream
    for given in ("loss", "m", "Z", "dlogits"):
        outs = {name: torch.full((T,), 5.0, device="cuda") for name in ("loss", "m", "Z")}
        buffer = torch.full((T * (V + 7),), 5.0, device="cuda")
        rows = buffer.view(T, V + 7)[:, 2:V + 2]
        status = _lib.load().more_distill(
            logits.data_ptr(), 32, T, V, V + 2, ids.data_ptr(), values.data_ptr(), k, tau, w.data_ptr(),
            *[outs[name].data_ptr() if name == given else None for name in ("loss", "m", "Z")],
            rows.data_ptr() if given == "dlogits" else None, V + 7, stream)
        assert status == _lib.OK
        for name, t in outs.items():
            assert torch.equal(t, getattr(want, name)) if name == given else (t == 5).all()
        if given == "dlogits":
            assert torch.equal(rows, want.dlogits)
            rows[:] = 5
        assert (buffer == 5).all()
