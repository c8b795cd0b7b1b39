"""The experts' linear maps against their 64-bit forms: every form of the kernels, ragged groups, dropped entries."""
import numpy as np
import pytest

import linear_ref as ref
from gpu_util import announce, require_gpu, to_dev
from layer_ref import dispatch, from_bf16, to_bf16

pytestmark = pytest.mark.gpu


def selection(rng, T, M, k, drop, hot=False):
    idx = rng.integers(0, M, (T, k)).astype(np.int32)
    if hot:
        idx[: 3 * T // 4] = M // 2  # (one expert has most entries; a token has it k times)
    if drop:
        out = rng.random((T, k)) < drop
        idx[out] = rng.choice([-1, M, 2 ** 31 - 1, -(2 ** 31)], out.sum()).astype(np.int32)
    return idx


def case(seed, T, K, N, M, k, drop=0.1, hot=False):
    rng = np.random.default_rng(seed)
    x = to_bf16(rng.standard_normal((T, K)))
    W = to_bf16(rng.standard_normal((M, N, K)) * K ** -0.5)
    dy = to_bf16(rng.standard_normal((T * k, N)))
    idx = selection(rng, T, M, k, drop, hot)
    return x, W, dy, idx, *dispatch(idx, M)


def within(got, want, bound, what):
    worst = np.max(np.abs(got - want) / bound) if got.size else 0.0
    assert worst <= 1.0, "%s is %.3g times its bound off" % (what, worst)


def to_np(t):
    import torch
    t = t.contiguous()
    return from_bf16(t.view(torch.uint16).cpu().numpy()) if t.dtype == torch.bfloat16 else t.cpu().numpy().astype(np.float64)


# (T, K, N, M, k): single tokens, odd sizes, a contraction of one piece, wide and narrow results, dense maps, tiles of
# every size
SHAPES = [(1, 2048, 128, 64, 8), (1, 8, 8, 1, 1), (3, 24, 40, 5, 2), (37, 72, 8, 11, 3), (64, 520, 264, 7, 1),
          (300, 136, 144, 9, 6), (129, 64, 512, 40, 1), (513, 256, 96, 3, 2), (2000, 200, 328, 4, 1), (1500, 72, 56, 300, 4),
          (1, 4096, 1032, 2, 1), (16, 1024, 72, 1, 1), (700, 640, 640, 1, 1), (5000, 64, 64, 2, 1), (40, 16, 2056, 33, 32)]


@pytest.mark.parametrize("T,K,N,M,k", SHAPES)
def test_linear(T, K, N, M, k):
    torch = require_gpu()
    from paper_2609_36301_amd import expert_linear, expert_linear_plan
    x, W, _, idx, offsets, srt = case(T + K, T, K, N, M, k)
    for bits, dtype in ((16, torch.bfloat16), (32, torch.float32)):
        announce("expert_linear T=%d K=%d N=%d M=%d k=%d bits=%d %s" % (T, K, N, M, k, bits, expert_linear_plan(T, K, N, M, k)))
        y = expert_linear(to_dev(x), to_dev(W), to_dev(idx), to_dev(offsets), to_dev(srt), out_dtype=dtype)
        want, bound = ref.linear(from_bf16(x), from_bf16(W), idx, bits)
        within(to_np(y), want, bound, "y")
        dropped = (idx.ravel() < 0) | (idx.ravel() >= M)
        assert not to_np(y)[dropped].any()


@pytest.mark.parametrize("T,K,N,M,k", SHAPES)
def test_linear_backward(T, K, N, M, k):
    require_gpu()
    from paper_2609_36301_amd import expert_linear_backward, expert_linear_plan
    x, W, dy, idx, offsets, srt = case(T + N, T, K, N, M, k)
    announce("expert_linear_backward T=%d K=%d N=%d M=%d k=%d %s" % (T, K, N, M, k, expert_linear_plan(T, K, N, M, k, "backward")))
    args = [to_dev(v) for v in (x, W, idx, offsets, srt, dy)]
    g = expert_linear_backward(*args)
    (dx, dW), (bx, bW) = ref.linear_backward(from_bf16(x), from_bf16(W), idx, from_bf16(dy))
    within(to_np(g.dx), dx, bx, "dx")
    within(to_np(g.dWt), dW, bW, "dW")
    one = expert_linear_backward(*args, need_dW=False)
    two = expert_linear_backward(*args, need_dx=False)
    assert one.dWt is None and two.dx is None
    assert (one.dx == g.dx).all() and (two.dWt == g.dWt).all()


# every form of the kernels: the smallest shape of a grid that the rules give it
FORMS = [{"tile_rows": 0, "cols": 16}, {"tile_rows": 0, "cols": 256}, {"tile_rows": 32, "cols": 64},
         {"tile_rows": 32, "cols": 128, "stages": 3}, {"tile_rows": 32, "cols": 128, "stages": 2},
         {"tile_rows": 64, "cols": 64}, {"tile_rows": 64, "cols": 128}, {"tile_rows": 128, "cols": 64},
         {"tile_rows": 128, "cols": 128}, {"tile_rows": 256, "cols": 256}]
DX_FORMS = [{"tile_rows": rows, "cols": cols} for rows in (32, 64, 128) for cols in (64, 128)] + [{"tile_rows": 256, "cols": 256}]
DW_FORMS = [{"dw_rows": r, "dw_cols": c, "dw_runs": n} for r, c in ((128, 128), (128, 64), (64, 128)) for n in (1, 2, 8, 32)]
DW_FORMS += [{"dw_rows": 256, "dw_cols": 256, "dw_runs": 1}]


def smallest(form, kind, entries=None, deep=False):
    """(T, K, N, M, k) of least work whose plan has these fields; deep: with a contraction of many stages."""
    from paper_2609_36301_amd import expert_linear_plan
    best = None
    for n in (40, 300, 2300, 9000, 33000):
        for M in (1, 3, 20, 150, 1500):
            for k in (1, 2):
                if entries is not None and k != entries:
                    continue
                for K in (48, 144, 528, 1040, 2064):
                    for N in (24, 136, 520, 1032, 2056):
                        if deep and (K < 528 if kind != "backward" else N < 520):
                            continue
                        work = n * K * N + 40 * M * K * N
                        if best and best[0] <= work:
                            continue
                        plan = expert_linear_plan(n // k, K, N, M, k, kind)
                        if all(plan[f] == v for f, v in form.items()):
                            best = work, (n // k, K, N, M, k), plan
    assert best, "no shape of the grid has the form %s" % form
    return best[1], best[2]


@pytest.mark.parametrize("deep", [False, True])
@pytest.mark.parametrize("form", FORMS, ids=str)
def test_linear_forms(form, deep):
    torch = require_gpu()
    from paper_2609_36301_amd import expert_linear
    # (without tiles, a workgroup takes 256 columns only of short contractions)
    (T, K, N, M, k), plan = smallest(form, "linear", deep=deep and form != {"tile_rows": 0, "cols": 256})
    x, W, _, idx, offsets, srt = case(T, T, K, N, M, k, hot=True)
    announce("expert_linear T=%d K=%d N=%d M=%d k=%d %s" % (T, K, N, M, k, plan))
    for bits, dtype in ((16, torch.bfloat16), (32, torch.float32)):
        y = expert_linear(to_dev(x), to_dev(W), to_dev(idx), to_dev(offsets), to_dev(srt), out_dtype=dtype)
        want, bound = ref.linear(from_bf16(x), from_bf16(W), idx, bits)
        within(to_np(y), want, bound, "y")


@pytest.mark.parametrize("entries,deep", [(1, False), (2, False), (1, True)])
@pytest.mark.parametrize("form", DX_FORMS + DW_FORMS, ids=str)
def test_linear_backward_forms(form, entries, deep):
    require_gpu()
    from paper_2609_36301_amd import expert_linear_backward
    # (64 rows of dW: N <= 64)
    (T, K, N, M, k), plan = smallest(form, "backward", entries, deep and form.get("dw_rows") != 64)
    x, W, dy, idx, offsets, srt = case(T, T, K, N, M, k, hot=True)
    announce("expert_linear_backward T=%d K=%d N=%d M=%d k=%d %s" % (T, K, N, M, k, plan))
    g = expert_linear_backward(*[to_dev(v) for v in (x, W, idx, offsets, srt, dy)])
    (dx, dW), (bx, bW) = ref.linear_backward(from_bf16(x), from_bf16(W), idx, from_bf16(dy))
    within(to_np(g.dx), dx, bx, "dx")
    within(to_np(g.dWt), dW, bW, "dW")


@pytest.mark.parametrize("drop", [1.0, 0.0])
def test_all_dropped_and_none(drop):
    require_gpu()
    from paper_2609_36301_amd import expert_linear, expert_linear_backward
    T, K, N, M, k = 70, 64, 72, 5, 3
    x, W, dy, idx, offsets, srt = case(7, T, K, N, M, k, drop=drop)
    announce("expert_linear, share dropped %g" % drop)
    args = [to_dev(v) for v in (x, W, idx, offsets, srt)]
    y, g = expert_linear(*args), expert_linear_backward(*args, to_dev(dy))
    if drop == 1.0:
        assert not to_np(y).any() and not to_np(g.dx).any() and not to_np(g.dWt).any()
    else:
        within(to_np(y), *ref.linear(from_bf16(x), from_bf16(W), idx), "y")


def test_no_tokens():
    torch = require_gpu()
    from paper_2609_36301_amd import expert_linear, expert_linear_backward, expert_linear_q8, quantize_rows
    x, W, dy, idx, offsets, srt = (to_dev(v) for v in case(1, 0, 16, 8, 3, 2))
    announce("no tokens")
    assert expert_linear(x, W, idx, offsets, srt).shape == (0, 8)
    g = expert_linear_backward(x, W, idx, offsets, srt, dy)
    assert g.dx.shape == (0, 16) and not to_np(g.dWt).any()
    q = quantize_rows(x)
    Wq = quantize_rows(W)
    assert expert_linear_q8(q.q, q.scale, Wq.q, Wq.scale, idx, offsets, srt).shape == (0, 8)
    torch.cuda.synchronize()


def test_rows_of_infinities_stay_in_their_rows():
    """What a row holds reaches that row's results alone, in tiles too."""
    require_gpu()
    from paper_2609_36301_amd import expert_linear
    T, K, N, M, k = 200, 136, 136, 2, 1
    x, W, _, idx, offsets, srt = case(3, T, K, N, M, k, drop=0)
    plain, bound = ref.linear(from_bf16(x), from_bf16(W), idx)
    x[17] = 0x7F80  # infinity
    x[90, 3] = 0x7FC0  # NaN
    announce("expert_linear with infinities and NaN in two rows")
    y = to_np(expert_linear(*[to_dev(v) for v in (x, W, idx, offsets, srt)]))
    other = np.ones(T, bool)
    other[[17, 90]] = False
    within(y[other], plain[other], bound[other], "y")
    assert not np.isfinite(y[17]).any() and np.isnan(y[90]).all()


def test_guards_around_outputs():
    """Nothing outside the outputs is written: they lie in larger buffers."""
    torch = require_gpu()
    from paper_2609_36301_amd import linear
    for T, K, N, M, k in ((3, 24, 40, 5, 2), (301, 72, 136, 9, 3), (5000, 64, 72, 2, 1)):
        x, W, dy, idx, offsets, srt = (to_dev(v) for v in case(T, T, K, N, M, k))
        announce("guards T=%d K=%d N=%d M=%d k=%d" % (T, K, N, M, k))

        def guarded(shape):
            n = int(np.prod(shape))
            big = torch.full((n + 256,), 7.0, dtype=torch.bfloat16, device="cuda")
            return big, big[128:128 + n].view(shape)

        f, b = linear.ExpertLinear(T, K, N, M, k), linear.ExpertLinearBackward(T, K, N, M, k)
        bufs = []
        for obj, name in ((f, "y"), (b, "dx"), (b, "dWt")):
            big, view = guarded(getattr(obj, name).shape)
            setattr(obj, name, view)
            bufs.append(big)
        f(x, W, idx, offsets, srt)
        b(x, W, idx, offsets, srt, dy)
        for big in bufs:
            assert (big[:128] == 7).all() and (big[-128:] == 7).all()


@pytest.mark.parametrize("M", [1, 2, 5, 255, 256, 257, 513, 1023, 1024, 1025])
@pytest.mark.parametrize("hot", [False, True])
def test_tiles_found_and_listed(M, hot):
    """Workgroups find their tiles among up to 1024 experts, of which many are empty or one has most entries, and dropped ones."""
    torch = require_gpu()
    from paper_2609_36301_amd import expert_linear, expert_linear_backward, expert_linear_plan, expert_linear_q8
    seen = set()
    for T, K, N, k in ((1700, 64, 72, 2), (611, 48, 264, 3), (9000, 16, 136, 1), (20000, 80, 8, 1)):
        plan = expert_linear_plan(T, K, N, M, k)
        seen.add((plan["tile_rows"], plan["listed"]))
        x, W, dy, idx, offsets, srt = case(M, T, K, N, M, k, hot=hot)
        announce("expert_linear of %d experts T=%d K=%d N=%d k=%d hot=%s %s" % (M, T, K, N, k, hot, plan))
        args = [to_dev(v) for v in (x, W, idx, offsets, srt)]
        within(to_np(expert_linear(*args)), *ref.linear(from_bf16(x), from_bf16(W), idx), "y")
        g = expert_linear_backward(*args, to_dev(dy))
        (dx, dW), (bx, bW) = ref.linear_backward(from_bf16(x), from_bf16(W), idx, from_bf16(dy))
        within(to_np(g.dx), dx, bx, "dx")
        within(to_np(g.dWt), dW, bW, "dW")
        q, Wq = (torch.from_numpy(np.random.default_rng(M).integers(-128, 128, s).astype(np.int8)) for s in ((T, K), (M, N, K)))
        qs, ws = np.full(T, 0.5, np.float32), np.full((M, N), 0.25, np.float32)
        y = expert_linear_q8(q.cuda(), to_dev(qs), Wq.cuda(), to_dev(ws), *args[2:])
        want, bound = ref.linear_q8(q.numpy(), qs.astype(np.float64), Wq.numpy(), ws.astype(np.float64), idx)
        within(to_np(y), want, bound, "y of 8 bits")
    assert any(rows and not listed for rows, listed in seen) == (M <= 1024)


@pytest.mark.parametrize("T,K,N,M,k", [(9000, 72, 264, 1500, 1), (5000, 128, 520, 1100, 2), (40000, 40, 520, 1200, 1), (30000, 528, 56, 1200, 1),
                                       (20000, 128, 136, 1300, 3), (260000, 72, 136, 2, 1), (130000, 72, 136, 2, 2)])
def test_gradients_of_many_small_experts(T, K, N, M, k):
    """Narrow tiles of dW with one stage, tiles along N (in runs, too), several tiles to a workgroup, experts of none to several
    stages."""
    require_gpu()
    from paper_2609_36301_amd import expert_linear_backward, expert_linear_plan
    for hot in (False, True):
        x, W, dy, idx, offsets, srt = case(K + N, T, K, N, M, k, hot=hot)
        announce("expert_linear_backward T=%d K=%d N=%d M=%d k=%d hot=%s %s"
                 % (T, K, N, M, k, hot, expert_linear_plan(T, K, N, M, k, "backward")))
        g = expert_linear_backward(*[to_dev(v) for v in (x, W, idx, offsets, srt, dy)])
        (dx, dW), (bx, bW) = ref.linear_backward(from_bf16(x), from_bf16(W), idx, from_bf16(dy))
        within(to_np(g.dx), dx, bx, "dx")
        within(to_np(g.dWt), dW, bW, "dW")


@pytest.mark.parametrize("M", [65537, 70000])
def test_more_experts_than_one_list_counts(M):
    """Beyond 2^16 experts their tiles are counted ahead of the list."""
    require_gpu()
    from paper_2609_36301_amd import expert_linear, expert_linear_backward, expert_linear_plan
    T, K, N, k = 1500, 16, 16, 2
    assert expert_linear_plan(T, K, N, M, k)["tile_rows"]
    x, W, dy, idx, offsets, srt = case(M, T, K, N, M, k)
    announce("expert_linear of %d experts" % M)
    args = [to_dev(v) for v in (x, W, idx, offsets, srt)]
    within(to_np(expert_linear(*args)), *ref.linear(from_bf16(x), from_bf16(W), idx), "y")
    g = expert_linear_backward(*args, to_dev(dy))
    (dx, dW), (bx, bW) = ref.linear_backward(from_bf16(x), from_bf16(W), idx, from_bf16(dy))
    within(to_np(g.dx), dx, bx, "dx")
    within(to_np(g.dWt), dW, bW, "dW")


def test_offsets_and_sorted_of_another_selection():
    """Values are undefined then; nothing outside the buffers is touched (the kernels' own checks), and every call ends."""
    torch = require_gpu()
    from paper_2609_36301_amd import linear
    rng = np.random.default_rng(8)
    for T, K, N, M, k in ((5, 32, 24, 4, 2), (300, 144, 136, 9, 3), (9000, 2064, 520, 3, 1)):
        x, W, dy, idx, offsets, srt = case(T, T, K, N, M, k)
        n = T * k
        wild = rng.integers(-2 ** 31, 2 ** 31, M + 1).astype(np.int32)
        near = rng.integers(-3, n + 4, M + 1).astype(np.int32)
        for o, s in ((wild, srt), (near, srt), (np.zeros_like(offsets), srt), (np.full_like(offsets, n), srt),
                     (offsets, rng.integers(-2 ** 31, 2 ** 31, n).astype(np.int32)), (offsets[::-1].copy(), np.zeros_like(srt))):
            announce("other offsets and sorted T=%d K=%d N=%d M=%d k=%d" % (T, K, N, M, k))
            f, b = linear.ExpertLinear(T, K, N, M, k), linear.ExpertLinearBackward(T, K, N, M, k)
            q = linear.ExpertLinearQ8(T, K, N, M, k)
            bufs = []
            for obj, name in ((f, "y"), (q, "y"), (b, "dx"), (b, "dWt")):
                size = getattr(obj, name).numel()
                big = torch.full((size + 256,), 7.0, dtype=torch.bfloat16, device="cuda")
                setattr(obj, name, big[128:128 + size].view(getattr(obj, name).shape))
                bufs.append(big)
            f(to_dev(x), to_dev(W), to_dev(idx), to_dev(o), to_dev(s))
            b(to_dev(x), to_dev(W), to_dev(idx), to_dev(o), to_dev(s), to_dev(dy))
            ones = lambda *shape: torch.ones(shape, device="cuda")  # noqa: E731
            eights = lambda *shape: torch.ones(shape, device="cuda", dtype=torch.int8)  # noqa: E731
            q(eights(T, K), ones(T), eights(M, N, K), ones(M, N), to_dev(idx), to_dev(o), to_dev(s), ones(T, k))
            torch.cuda.synchronize()
            for big in bufs:
                assert (big[:128] == 7).all() and (big[-128:] == 7).all()


def test_calls_without_a_workspace():
    """Where none is needed it may be NULL."""
    torch = require_gpu()
    from paper_2609_36301_amd import _lib, expert_linear, expert_linear_backward, linear
    T, K, N, M, k = 400, 72, 40, 20, 1
    assert linear.expert_linear_workspace_size(T, K, N, M, k) == linear.expert_linear_backward_workspace_size(T, K, N, M, k) == 0
    announce("expert_linear and its backward pass without a workspace")
    args = [to_dev(v) for v in case(4, T, K, N, M, k)]
    x, W, dy, idx, offsets, srt = args
    y, dx, dW = (torch.full(s, 7.0, dtype=torch.bfloat16, device="cuda") for s in ((T, N), (T, K), (M, N, K)))
    lib, stream = _lib.load(), torch.cuda.current_stream().cuda_stream
    head = [x.data_ptr(), W.data_ptr(), T, K, N, M, k, idx.data_ptr(), offsets.data_ptr(), srt.data_ptr()]
    assert lib.more_expert_linear(*head, y.data_ptr(), 16, None, 0, stream) == _lib.OK
    assert lib.more_expert_linear_backward(*head, dy.data_ptr(), dx.data_ptr(), dW.data_ptr(), None, 0, stream) == _lib.OK
    g = expert_linear_backward(x, W, idx, offsets, srt, dy)
    assert torch.equal(y, expert_linear(x, W, idx, offsets, srt)) and torch.equal(dx, g.dx) and torch.equal(dW, g.dWt)


def test_same_bits_every_run():
    require_gpu()
    from paper_2609_36301_amd import expert_linear, expert_linear_backward
    for T, K, N, M, k in ((500, 136, 264, 3, 4), (9000, 64, 72, 1, 1)):
        args = [to_dev(v) for v in case(11, T, K, N, M, k)]
        x, W, dy, idx, offsets, srt = args
        announce("repeats T=%d" % T)
        first = None
        for _ in range(4):
            g = expert_linear_backward(x, W, idx, offsets, srt, dy)
            got = [t.clone() for t in (expert_linear(x, W, idx, offsets, srt), g.dx, g.dWt)]
            first = first or got
            assert all((a.view(a.shape) == b).all() for a, b in zip(got, first))


# ------------------------------------------------------------------------------ 8 bits
Q8_SHAPES = [(1, 2048, 128, 64, 8), (1, 16, 8, 1, 1), (3, 48, 40, 5, 2), (37, 144, 8, 11, 3), (64, 1040, 264, 7, 1),
             (300, 272, 144, 9, 6), (129, 128, 512, 40, 1), (2000, 400, 328, 4, 1), (1500, 144, 56, 300, 4), (16, 4096, 72, 1, 1)]


@pytest.mark.parametrize("T,K,N,M,k", Q8_SHAPES)
def test_linear_q8(T, K, N, M, k):
    q8_case(T, K, N, M, k)


@pytest.mark.parametrize("deep", [False, True])
@pytest.mark.parametrize("form", FORMS, ids=str)
def test_linear_q8_forms(form, deep):
    q8_case(*smallest(form, "q8", deep=deep and form != {"tile_rows": 0, "cols": 256})[0])


def q8_case(T, K, N, M, k):
    torch = require_gpu()
    from paper_2609_36301_amd import expert_linear_plan, expert_linear_q8
    rng = np.random.default_rng(T + K)
    q = rng.integers(-128, 128, (T, K)).astype(np.int8)
    Wq = rng.integers(-128, 128, (M, N, K)).astype(np.int8)
    if T > 2:
        q[0], Wq[0] = -128, -128  # the largest sums
    qs, ws = (rng.random(T) + 0.01).astype(np.float32), (rng.random((M, N)) + 0.01).astype(np.float32)
    gate = rng.standard_normal((T, k)).astype(np.float32)
    idx = selection(rng, T, M, k, 0.1, hot=T > 1000)
    idx[0, 0] = 0
    gate.ravel()[(idx.ravel() < 0) | (idx.ravel() >= M)] = np.nan  # (not read)
    offsets, srt = dispatch(idx, M)
    for bits, dtype, g in ((16, torch.bfloat16, gate), (32, torch.float32, None)):
        announce("expert_linear_q8 T=%d K=%d N=%d M=%d k=%d bits=%d %s"
                 % (T, K, N, M, k, bits, expert_linear_plan(T, K, N, M, k, "q8")))
        y = expert_linear_q8(*[to_dev(v) for v in (q, qs, Wq, ws, idx, offsets, srt)], None if g is None else to_dev(g),
                             out_dtype=dtype)
        want, bound = ref.linear_q8(q, qs.astype(np.float64), Wq, ws.astype(np.float64), idx,
                                    None if g is None else g.astype(np.float64), bits)
        within(to_np(y), want, bound, "y")


def test_q8_largest_sums():
    """65536 products of (-128)^2: 2^30, exact in the sum's 32 bits; tiles and the kernel without them."""
    torch = require_gpu()
    from paper_2609_36301_amd import expert_linear_q8
    K, N, M = 65536, 264, 1
    for T in (3, 700):
        announce("expert_linear_q8 T=%d K=%d N=%d, largest sums" % (T, K, N))
        q = torch.full((T, K), -128, dtype=torch.int8, device="cuda")
        Wq = torch.full((M, N, K), -128, dtype=torch.int8, device="cuda")
        q[T - 1, 5] = 127
        idx = np.zeros((T, 1), np.int32)
        offsets, srt = dispatch(idx, M)
        y = expert_linear_q8(q, torch.ones(T, device="cuda"), Wq, torch.ones((M, N), device="cuda"), to_dev(idx), to_dev(offsets),
                             to_dev(srt), out_dtype=torch.float32)
        assert (y[:T - 1] == 2.0 ** 30).all() and (y[T - 1] == 2.0 ** 30 - 128 * 255).all()


def test_q8_bad_rows_are_nan_and_alone():
    torch = require_gpu()
    from paper_2609_36301_amd import expert_linear_q8, quantize_rows
    T, K, N, M = 40, 64, 24, 3
    rng = np.random.default_rng(5)
    x = to_bf16(rng.standard_normal((T, K)))
    x[4, 7], x[9] = 0x7F80, 0
    W = quantize_rows(to_dev(to_bf16(rng.standard_normal((M, N, K)))))
    idx = selection(rng, T, M, 1, 0)
    offsets, srt = dispatch(idx, M)
    announce("expert_linear_q8 with an infinite row and a row of zeros")
    r = quantize_rows(to_dev(x))
    y = to_np(expert_linear_q8(r.q, r.scale, W.q, W.scale, to_dev(idx), to_dev(offsets), to_dev(srt)))
    assert np.isnan(y[4]).all() and not y[9].any() and np.isfinite(np.delete(y, 4, axis=0)).all()
    torch.cuda.synchronize()


# ------------------------------------------------------------------------------ rows in 8 bits
WIDTHS = [16, 48, 512, 528, 1024, 1040, 2048, 2064, 8192, 8208, 32768, 32784, 65536]


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("T", [1, 5, 70])
def test_quantize_rows_to_the_bit(width, T):
    require_gpu()
    from paper_2609_36301_amd import quantize_rows
    rng = np.random.default_rng(width + T)
    x = rng.standard_normal((T, width)) * np.exp(rng.uniform(-8, 8, (T, 1)))
    x[0, :3] = [4.0, 2.0, -2.0]
    x = to_bf16(x)
    if T > 4:
        x[1] = 0
        x[2, width - 1] = 0xFF80
        x[3, 0] = 0x7FC1
        x[4] = to_bf16(np.full(width, 2.0 ** -101))
        x[4, 5] = 0x8001  # a denormal
    announce("quantize_rows T=%d width=%d" % (T, width))
    r = quantize_rows(to_dev(x))
    q, scale = ref.quantize(from_bf16(x))
    assert np.array_equal(r.q.cpu().numpy(), q)
    assert np.array_equal(r.scale.cpu().numpy(), scale, equal_nan=True)


@pytest.mark.parametrize("width", [16, 528, 1040, 2064, 8208, 65536])
def test_quantize_gated_rows(width):
    """Off by at most half a step of the row, and by what fp32 is off before."""
    require_gpu()
    from paper_2609_36301_amd import quantize_rows
    rng = np.random.default_rng(width)
    x = to_bf16(3 * rng.standard_normal((9, 2 * width)))
    x[3, :width] = to_bf16(np.full(width, -200.0))  # silu vanishes
    x[5, 1] = 0x7F80
    announce("quantize_rows gated width=%d" % width)
    r = quantize_rows(to_dev(x), gated=True)
    q, scale = r.q.cpu().numpy().astype(np.float64), r.scale.cpu().numpy().astype(np.float64)
    with np.errstate(all="ignore"):
        v, err = ref.gated(from_bf16(x))
    rows = np.array([i for i in range(9) if i not in (3, 5)])
    a = np.abs(v[rows]).max(axis=1)
    assert (np.abs(scale[rows] - a / 127) <= (err[rows].max(axis=1) + 2 * ref.E32 * a) / 127).all()
    off = np.abs(q[rows] * scale[rows, None] - v[rows])
    assert (off <= 0.5 * scale[rows, None] * (1 + 1e-6) + 4 * err[rows].max(axis=1, keepdims=True)).all()
    assert np.abs(q[rows]).max() == 127
    assert scale[3] == 0 and not q[3].any() and np.isnan(scale[5]) and not q[5].any()


def test_quantize_leading_dimensions():
    require_gpu()
    from paper_2609_36301_amd import quantize_rows
    rng = np.random.default_rng(9)
    W = to_bf16(rng.standard_normal((3, 5, 32)))
    announce("quantize_rows of weights")
    r = quantize_rows(to_dev(W))
    q, scale = ref.quantize(from_bf16(W).reshape(15, 32))
    assert r.q.shape == (3, 5, 32) and r.scale.shape == (3, 5)
    assert np.array_equal(r.q.cpu().numpy().reshape(15, 32), q) and np.array_equal(r.scale.cpu().numpy().ravel(), scale)
