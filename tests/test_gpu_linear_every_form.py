"""Every form of the linear maps and of their gradients, alone and in one launch, on a small shape and on a larger one, into
outputs full of NaN: what a call leaves unwritten is seen."""
import numpy as np
import pytest

import linear_forms
import linear_ref as ref
from gpu_util import announce, require_gpu, to_dev
from layer_ref import dispatch, from_bf16
from test_gpu_linear import case, selection, to_np, within

pytestmark = pytest.mark.gpu

FORWARD = [f for f in linear_forms.expected() if f[0] == "linear"]
Q8 = [f for f in linear_forms.expected() if f[0] == "q8"]
BACKWARD = [f for f in linear_forms.expected() if f[0] in ("dx", "dW", "both")]
NAN = float("nan")


def shapes_of(form):
    return [(hot, *shape) for hot, shape in zip((False, True), linear_forms.shapes()[form])]


def check(got, want, bound, what):
    got = to_np(got)
    assert np.isfinite(got).all(), "%s: %d elements were not written" % (what, (~np.isfinite(got)).sum())
    within(got, want, bound, what)


@pytest.mark.parametrize("form", FORWARD, ids=linear_forms.ids)
def test_linear(form):
    torch = require_gpu()
    from paper_2609_36301_amd import linear
    for hot, T, K, N, M, k in shapes_of(form):
        x, W, _, idx, offsets, srt = case(T + K, T, K, N, M, k, hot=hot)
        args = [to_dev(v) for v in (x, W, idx, offsets, srt)]
        for bits, dtype in ((16, torch.bfloat16), (32, torch.float32)):
            announce("expert_linear %s T=%d K=%d N=%d M=%d k=%d bits=%d" % (linear_forms.ids(form), T, K, N, M, k, bits))
            call = linear.ExpertLinear(T, K, N, M, k, out_dtype=dtype)
            call.y.fill_(NAN)
            check(call(*args), *ref.linear(from_bf16(x), from_bf16(W), idx, bits), "y")


@pytest.mark.parametrize("form", Q8, ids=linear_forms.ids)
def test_linear_q8(form):
    torch = require_gpu()
    from paper_2609_36301_amd import linear
    for hot, T, K, N, M, k in shapes_of(form):
        rng = np.random.default_rng(T + K)
        q, Wq = (rng.integers(-128, 128, s).astype(np.int8) for s in ((T, K), (M, N, K)))
        qs, ws = (rng.random(T) + 0.01).astype(np.float32), (rng.random((M, N)) + 0.01).astype(np.float32)
        gate = rng.standard_normal((T, k)).astype(np.float32)
        idx = selection(rng, T, M, k, 0.1, hot)
        given = [to_dev(v) for v in (q, qs, Wq, ws, idx, *dispatch(idx, M))]
        for bits, dtype, g in ((16, torch.bfloat16, gate), (32, torch.float32, None)):
            announce("expert_linear_q8 %s T=%d K=%d N=%d M=%d k=%d bits=%d" % (linear_forms.ids(form), T, K, N, M, k, bits))
            call = linear.ExpertLinearQ8(T, K, N, M, k, out_dtype=dtype)
            call.y.fill_(NAN)
            y = call(*given, None if g is None else to_dev(g))
            check(y, *ref.linear_q8(q, qs.astype(np.float64), Wq, ws.astype(np.float64), idx,
                                    None if g is None else g.astype(np.float64), bits), "y")


@pytest.mark.parametrize("form", BACKWARD, ids=linear_forms.ids)
def test_gradients(form):
    require_gpu()
    from paper_2609_36301_amd import linear
    for hot, T, K, N, M, k in shapes_of(form):
        x, W, dy, idx, offsets, srt = case(T + N, T, K, N, M, k, hot=hot)
        announce("expert_linear_backward %s T=%d K=%d N=%d M=%d k=%d" % (linear_forms.ids(form), T, K, N, M, k))
        call = linear.ExpertLinearBackward(T, K, N, M, k, need_dx=form[0] != "dW", need_dW=form[0] != "dx")
        for out in (call.dx, call.dWt):
            if out is not None:
                out.fill_(NAN)
        if call.workspace_bytes:  # (fp32 NaN: shares and runs that are read must have been written)
            call.workspace.fill_(255)
        g = call(*[to_dev(v) for v in (x, W, idx, offsets, srt, dy)])
        (dx, dW), (bx, bW) = ref.linear_backward(from_bf16(x), from_bf16(W), idx, from_bf16(dy))
        if g.dx is not None:
            check(g.dx, dx, bx, "dx")
        if g.dWt is not None:
            check(g.dWt, dW, bW, "dW")


@pytest.mark.parametrize("T,K,N,M,k", [(70, 64, 72, 5, 3), (400, 72, 136, 9, 1), (9000, 64, 512, 1500, 2), (0, 16, 8, 3, 2)])
def test_everything_dropped(T, K, N, M, k):
    """Zeros, where NaN was."""
    require_gpu()
    from paper_2609_36301_amd import linear
    x, W, dy, idx, offsets, srt = (to_dev(v) for v in case(7, T, K, N, M, k, drop=1.0))
    announce("expert_linear, all dropped T=%d" % T)
    f, b = linear.ExpertLinear(T, K, N, M, k), linear.ExpertLinearBackward(T, K, N, M, k)
    for out in (f.y, b.dx, b.dWt):
        out.fill_(NAN)
    g = b(x, W, idx, offsets, srt, dy)
    assert (f(x, W, idx, offsets, srt) == 0).all() and (g.dx == 0).all() and (g.dWt == 0).all()


@pytest.mark.parametrize("T,K,N,M,k", [(3, 24, 40, 5, 2), (301, 72, 136, 9, 3), (500, 136, 264, 3, 4), (5000, 64, 72, 2, 1),
                                       (9000, 64, 72, 1, 1)])
def test_all_is_written_each_time_with_the_same_bits(T, K, N, M, k):
    """Between guards, over NaN, four times."""
    torch = require_gpu()
    from paper_2609_36301_amd import linear
    x, W, dy, idx, offsets, srt = case(T, T, K, N, M, k)
    announce("expert_linear and gradients between guards T=%d K=%d N=%d M=%d k=%d" % (T, K, N, M, k))
    args = [to_dev(v) for v in (x, W, idx, offsets, srt)]
    f, b = linear.ExpertLinear(T, K, N, M, k), linear.ExpertLinearBackward(T, K, N, M, k)
    bufs = []
    for obj, name in ((f, "y"), (b, "dx"), (b, "dWt")):
        out = getattr(obj, name)
        big = torch.full((out.numel() + 256,), 7.0, dtype=out.dtype, device="cuda")
        setattr(obj, name, big[128:128 + out.numel()].view(out.shape))
        bufs.append(big)
    (dx, dW), (bx, bW) = ref.linear_backward(from_bf16(x), from_bf16(W), idx, from_bf16(dy))
    y, by = ref.linear(from_bf16(x), from_bf16(W), idx)
    first = None
    for _ in range(4):
        for big in bufs:
            big[128:-128] = NAN
        f(*args)
        b(*args, to_dev(dy))
        got = [big.clone() for big in bufs]
        first = first or got
        assert all(torch.equal(a, c) for a, c in zip(got, first))
        assert all((big[:128] == 7).all() and (big[-128:] == 7).all() for big in bufs)
    check(f.y, y, by, "y")
    check(b.dx, dx, bx, "dx")
    check(b.dWt, dW, bW, "dW")
