"""Distillation from a teacher's top logits against its 64-bit form: every row length, odd strides, rows without a teacher,
masked logits."""
import math

import numpy as np
import pytest

import linear_ref as ref
from gpu_util import announce, require_gpu, to_dev
from layer_ref import from_bf16, to_bf16

pytestmark = pytest.mark.gpu


def case(seed, T, V, k, bits, spread=3.0):
    rng = np.random.default_rng(seed)
    z = rng.standard_normal((T, V)) * spread
    z = z.astype(np.float32).astype(np.float64) if bits == 32 else from_bf16(to_bf16(z))
    ids = rng.integers(0, V, (T, k)).astype(np.int32)  # (with repeats)
    ids[:, 0] = V - 1
    values = -np.sort(-rng.standard_normal((T, k)) * 2).astype(np.float32) + 3
    if T > 4:
        ids[1] = -1                     # no teacher
        ids[2, k // 2:] = V             # some of it
        values[3, k // 2:] = -np.inf
        ids[4] = 0                      # one class k times
    return z, ids, values, rng.standard_normal(T).astype(np.float32)


def rows_on_device(z, bits, ld=None, start=0):
    """z as rows that lie ld apart, `start` elements into a buffer of sevens."""
    import torch
    T, V = z.shape
    ld = V if ld is None else ld
    dtype = torch.float32 if bits == 32 else torch.bfloat16
    big = torch.full((start + T * ld + 8,), 7.0, dtype=dtype, device="cuda")
    view = big[start:start + T * ld].view(T, ld)[:, :V] if T * ld else big[:0].view(T, V)
    view.copy_(torch.from_numpy(z).to(dtype))
    return big, view


def close(got, want, bound, what):
    got = got.detach().double().cpu().numpy()
    worst = np.max(np.abs(got - want) / bound) if got.size else 0.0
    assert worst <= 1.0, "%s is %.3g times its bound off" % (what, worst)


# rows of every length: a piece or less, each form's last and the next form's first, rows that are read twice
LENGTHS = [1, 2, 7, 8, 9, 63, 250, 256, 505, 512, 1000, 1017, 1024, 2033, 2040, 2048, 4081, 4089, 8185, 8193, 16361, 16377,
           32753, 32761, 65513, 65529, 131049, 131065, 140001]


@pytest.mark.parametrize("bits", [16, 32])
@pytest.mark.parametrize("V", LENGTHS)
def test_distill(V, bits):
    torch = require_gpu()
    from paper_2609_36301_amd import distill_backward, distill_loss
    T, k, tau = (11, 5, 2.0) if V < 60000 else (6, 5, 2.0)
    z, ids, values, w = case(V, T, V, k, bits)
    for ld, start in ((V, 0), (V + 3, 1), ((V + 7) // 8 * 8, 0)):
        announce("distill V=%d bits=%d ld=%d start=%d" % (V, bits, ld, start))
        (loss, m, Z, grad), (bl, bZ, bg) = ref.distill(z, ids, values.astype(np.float64), tau, w.astype(np.float64), bits)
        big, logits = rows_on_device(z, bits, ld, start)
        d = distill_loss(logits, to_dev(ids), to_dev(values), to_dev(w), temperature=tau, gradient=True)
        close(d.loss, loss, bl, "loss")
        assert np.array_equal(d.m.cpu().numpy().astype(np.float64), m)
        close(d.Z, Z, bZ, "Z")
        close(d.dlogits, grad, bg, "dlogits")
        assert d.loss[1] == 0 and not d.dlogits[1].any()
        two = distill_backward(logits, d.m, d.Z, to_dev(ids), to_dev(values), to_dev(w), temperature=tau)
        assert torch.equal(two, d.dlogits)
        alone = distill_loss(logits, to_dev(ids), to_dev(values), temperature=tau)
        # (long rows are summed in another order without the gradient)
        close(alone.loss, loss, bl, "loss")
        close(alone.Z, Z, bZ, "Z")
        assert torch.equal(alone.m, d.m) and alone.dlogits is None


@pytest.mark.parametrize("bits", [16, 32])
@pytest.mark.parametrize("V,ld,start", [(9, 9, 0), (300, 301, 3), (1000, 1003, 5), (5000, 5001, 1), (20000, 20003, 1), (70001, 70001, 7),
                                        (140001, 140003, 3)])
def test_in_place_and_nothing_beside_the_rows(V, ld, start, bits):
    torch = require_gpu()
    from paper_2609_36301_amd import distill
    T, k, tau = 6, 4, 0.5
    z, ids, values, w = case(V, T, V, k, bits)
    dtype = torch.float32 if bits == 32 else torch.bfloat16
    announce("distill in place V=%d bits=%d ld=%d start=%d" % (V, bits, ld, start))
    _, logits = rows_on_device(z, bits, ld, start)
    args = to_dev(ids), to_dev(values)
    make = lambda **kw: distill.Distill(T, V, k, dtype=dtype, temperature=tau, ld=ld, gradient=True, **kw)  # noqa: E731
    out = make()
    buffer = torch.full((T * ld + 16,), 5.0, dtype=dtype, device="cuda")
    out.dlogits = buffer[8:8 + T * ld].view(T, ld)[:, :V]
    want = out(logits, *args, to_dev(w))
    want = (want.loss.clone(), want.m.clone(), want.Z.clone(), want.dlogits.clone())
    beside = torch.ones_like(buffer, dtype=torch.bool)
    beside[8:8 + T * ld].view(T, ld)[:, :V] = False
    assert (buffer[beside] == 5).all()
    for backward in (False, True):
        big, logits = rows_on_device(z, bits, ld, start)
        if backward:
            got = distill.DistillBackward(T, V, k, dtype=dtype, temperature=tau, ld=ld, inplace=True)(
                logits, want[1], want[2], *args, to_dev(w))
        else:
            got = make(inplace=True)(logits, *args, to_dev(w)).dlogits
        assert got.data_ptr() == logits.data_ptr() and torch.equal(got, want[3])
        beside = torch.ones_like(big, dtype=torch.bool)
        beside[start:start + T * ld].view(T, ld)[:, :V] = False
        assert (big[beside] == 7).all()


@pytest.mark.parametrize("bits", [16, 32])
@pytest.mark.parametrize("V,ld,start,ldd,start_d", [(13, 13, 0, 17, 1), (300, 304, 0, 301, 3), (3000, 3001, 5, 3008, 0), (9001, 9001, 3, 9008, 8),
                                                    (33000, 33000, 0, 33003, 1), (300001, 300001, 1, 300002, 5)])
def test_gradients_of_other_strides(V, ld, start, ldd, start_d, bits):
    """The library's call with gradients that lie otherwise than the logits."""
    torch = require_gpu()
    from paper_2609_36301_amd import _lib, distill_loss
    T, k, tau = 5, 3, 2.0
    z, ids, values, w = case(V, T, V, k, bits)
    announce("distill V=%d bits=%d gradients ldd=%d start=%d" % (V, bits, ldd, start_d))
    _, logits = rows_on_device(z, bits, ld, start)
    ids, values, w = to_dev(ids), to_dev(values), to_dev(w)
    want = distill_loss(logits, ids, values, w, temperature=tau, gradient=True)
    for given in (False, True):
        buffer = torch.full((T * ldd + 32,), 5.0, dtype=logits.dtype, device="cuda")
        rows = buffer[start_d:start_d + T * ldd].view(T, ldd)[:, :V]
        head = (logits.data_ptr(), bits, T, V, ld)
        entries = (ids.data_ptr(), values.data_ptr(), k, tau)
        tail = (rows.data_ptr(), ldd, torch.cuda.current_stream().cuda_stream)
        lib = _lib.load()
        if given:
            status = lib.more_distill_backward(*head, want.m.data_ptr(), want.Z.data_ptr(), *entries, w.data_ptr(), *tail)
        else:
            status = lib.more_distill(*head, *entries, w.data_ptr(), None, None, None, *tail)
        assert status == _lib.OK and torch.equal(rows, want.dlogits)
        beside = torch.ones_like(buffer, dtype=torch.bool)
        beside[start_d:start_d + T * ldd].view(T, ldd)[:, :V] = False
        assert (buffer[beside] == 5).all()


@pytest.mark.parametrize("tau", [2.0 ** -40, 2.0 ** 40])
def test_outermost_temperatures(tau):
    """Finite results; at the lowest the largest logit has all the probability, at the highest all classes have the same."""
    torch = require_gpu()
    from paper_2609_36301_amd import distill_loss
    T, V, k = 4, 700, 3
    announce("distill tau=%g" % tau)
    z = torch.zeros((T, V), device="cuda")
    z[:, 9] = 1.0
    ids = torch.tensor([[5, 9, 11]] * T, dtype=torch.int32, device="cuda")
    values = torch.tensor([[1.0, 0.0, -1.0]] * T, device="cuda")
    d = distill_loss(z, ids, values, temperature=tau, gradient=True)
    want = torch.zeros((T, V), dtype=torch.float64)
    if tau < 1:
        want[:, 9], want[:, 5] = tau, -tau
        loss = tau  # tau^2 (z_9 - z_5) / tau
    else:
        want[:] = tau / V
        want[:, [5, 9, 11]] -= tau / 3
        loss = tau * tau * math.log(V / 3)
    # a quotient of two fp32 numbers and a product: four roundings and two function values of 2^-21 each
    assert (d.dlogits.double().cpu() - want).abs().max() <= 2.0 ** -19 * tau
    assert (d.loss.double() - loss).abs().max() <= 2.0 ** -18 * loss


@pytest.mark.parametrize("k", [1, 63, 64, 65, 200, 1024])
def test_numbers_of_entries(k):
    require_gpu()
    from paper_2609_36301_amd import distill_loss
    for V in (700, 3000, 9000, 40000):
        z, ids, values, w = case(k + V, 7, V, k, 32)
        announce("distill V=%d k=%d" % (V, k))
        (loss, _, _, grad), (bl, _, bg) = ref.distill(z, ids, values.astype(np.float64), 1.5, w.astype(np.float64), 32)
        d = distill_loss(rows_on_device(z, 32)[1], to_dev(ids), to_dev(values), to_dev(w), temperature=1.5, gradient=True)
        close(d.loss, loss, bl, "loss")
        close(d.dlogits, grad, bg, "dlogits")


@pytest.mark.parametrize("V", [40, 600, 3000, 9000, 70000, 300000])
def test_masked_logits(V):
    """-infinity, and the type's lowest value, are classes without probability; whole pieces of them too."""
    require_gpu()
    from paper_2609_36301_amd import distill_loss
    T, k, tau = 6, 3, 1.0
    z, ids, values, w = case(V, T, V, k, 32)
    z[:, : V // 2] = -np.inf
    z[1, V // 2: V // 2 + 5] = np.finfo(np.float32).min
    z[5, :-1] = -np.inf  # one class is left
    ids[:] = np.random.default_rng(V).integers(V // 2 + 5, V, (T, k))
    ids[5] = V - 1
    ids[2, 1:], values[2, 1:] = 0, values[2, 0] - 1000  # an entry without weight on a masked class
    announce("distill with masked logits V=%d" % V)
    (loss, m, Z, grad), (bl, bZ, bg) = ref.distill(z, ids, values.astype(np.float64), tau, w.astype(np.float64), 32)
    d = distill_loss(rows_on_device(z, 32)[1], to_dev(ids), to_dev(values), to_dev(w), temperature=tau, gradient=True)
    assert np.isfinite(loss).all()
    close(d.loss, loss, bl, "loss")
    close(d.Z, Z, bZ, "Z")
    close(d.dlogits, grad, bg, "dlogits")


@pytest.mark.parametrize("V", [40, 3000, 20000, 300000])
def test_rows_that_have_no_loss_are_alone(V):
    torch = require_gpu()
    from paper_2609_36301_amd import distill_loss
    T, k = 6, 3
    z, ids, values, w = case(V, T, V, k, 32)
    ids[:] = np.arange(k)
    plain = z.copy()
    z[0] = -np.inf
    z[2, V // 3] = np.nan
    z[4, V // 2] = np.inf
    values[5, 0] = np.nan
    announce("distill with rows of NaN V=%d" % V)
    (loss, _, _, grad), (bl, _, bg) = ref.distill(plain, ids, values.astype(np.float64), 1.0, w.astype(np.float64), 32)
    d = distill_loss(rows_on_device(z, 32)[1], to_dev(ids), to_dev(values), to_dev(w), gradient=True)
    assert torch.isnan(d.loss[[0, 2, 4, 5]]).all()
    good = [1, 3]
    close(d.loss[good], loss[good], bl[good], "loss")
    close(d.dlogits[good], grad[good], bg[good], "dlogits")
    ids[:] = -1  # no teacher: no loss, whatever the student says
    d = distill_loss(rows_on_device(z, 32)[1], to_dev(ids), to_dev(values), to_dev(w), gradient=True)
    assert not d.loss.any() and not d.dlogits.any()


def test_large_logits_and_small_temperatures():
    require_gpu()
    from paper_2609_36301_amd import distill_loss
    for V in (100, 5000):
        for tau in (0.05, 20.0):
            z, ids, values, w = case(V, 8, V, 4, 32, spread=100.0)
            announce("distill V=%d tau=%g" % (V, tau))
            (loss, _, _, grad), (bl, _, bg) = ref.distill(z, ids, values.astype(np.float64), tau, w.astype(np.float64), 32)
            d = distill_loss(rows_on_device(z, 32)[1], to_dev(ids), to_dev(values), to_dev(w), temperature=tau, gradient=True)
            close(d.loss, loss, bl, "loss")
            close(d.dlogits, grad, bg, "dlogits")


def test_gradient_is_differences():
    """Of the kernel's own loss, along random directions: the loss is off by its bound at each end, the quotient of
    differences by the third derivative (below tau^-1 |direction|^3 here) times step^2 / 6."""
    require_gpu()
    from paper_2609_36301_amd import distill_loss
    rng = np.random.default_rng(4)
    T, V, k, tau, step = 8, 300, 4, 1.0, 2.0 ** -4
    z, ids, values, _ = case(5, T, V, k, 32, spread=1.0)
    announce("distill: differences")
    args = to_dev(ids), to_dev(values)
    d = distill_loss(rows_on_device(z, 32)[1], *args, temperature=tau, gradient=True)
    grad = d.dlogits.double().cpu().numpy()
    v = rng.standard_normal((T, V))
    v = np.rint(v / np.abs(v).max() * 256) / 256  # (the steps add up exactly in fp32)
    z0 = np.rint(z * 4096) / 4096
    grad = distill_loss(rows_on_device(z0, 32)[1], *args, temperature=tau, gradient=True).dlogits.double().cpu().numpy()
    ends = [distill_loss(rows_on_device(z0 + s * step * v, 32)[1], *args, temperature=tau).loss.double().cpu().numpy() for s in (1, -1)]
    _, (bl, _, bg) = ref.distill(z0, ids, values.astype(np.float64), tau, None, 32)
    off = np.abs((ends[0] - ends[1]) / (2 * step) - (grad * v).sum(1))
    assert (off <= 2 * bl / (2 * step) + (bg * np.abs(v)).sum(1) + step ** 2 / 6).all()


def test_no_rows():
    torch = require_gpu()
    from paper_2609_36301_amd import distill_loss
    announce("distill without rows")
    e = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    d = distill_loss(e(0, 50), e(0, 3, dtype=torch.int32), e(0, 3), gradient=True)
    assert d.loss.shape == (0,) and d.dlogits.shape == (0, 50)


@pytest.mark.parametrize("V", [64, 900, 5000, 20000, 70000, 140000])
@pytest.mark.parametrize("k", [32, 64, 200])
def test_entries_that_meet(V, k):
    """Entries next to one another, at a row's ends and more than once: each class has one gradient, of all its entries."""
    torch = require_gpu()
    from paper_2609_36301_amd import distill_loss
    T, tau = 9, 2.0
    for bits in (16, 32):
        z, ids, values, w = case(V + k, T, V, k, bits)
        rng = np.random.default_rng(V)
        near = np.r_[np.arange(20), np.arange(V - 20, V)]
        ids[:] = rng.choice(near, (T, k))
        ids[3] = V // 2
        ids[4, ::2] = -1
        announce("distill V=%d k=%d bits=%d, entries that meet" % (V, k, bits))
        (loss, _, _, grad), (bl, _, bg) = ref.distill(z, ids, values.astype(np.float64), tau, w.astype(np.float64), bits)
        logits = rows_on_device(z, bits, V + 1, 1)[1]
        d = distill_loss(logits, to_dev(ids), to_dev(values), to_dev(w), temperature=tau, gradient=True)
        close(d.loss, loss, bl, "loss")
        close(d.dlogits, grad, bg, "dlogits")
        again = distill_loss(logits, to_dev(ids), to_dev(values), to_dev(w), temperature=tau, gradient=True)
        assert torch.equal(again.dlogits, d.dlogits)
