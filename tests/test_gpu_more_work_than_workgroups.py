"""Calls whose rows, tiles or experts exceed the largest grid, so that a workgroup takes several one after the other."""
import pytest

from gpu_util import announce, require_gpu

pytestmark = pytest.mark.gpu

E16, E32 = 2.0 ** -8, 2.0 ** -24


@pytest.mark.parametrize("T,V,k", [((1 << 22) + 5, 5, 1), ((1 << 20) + 3, 4200, 3)])
def test_distillation(T, V, k):
    """Rows that repeat: each has the result that it has alone."""
    torch = require_gpu()
    from paper_2609_36301_amd import distill_backward, distill_loss
    announce("distill T=%d V=%d k=%d" % (T, V, k))
    gen = torch.Generator(device="cuda").manual_seed(5)
    some = 7
    z = torch.randn((some, V), device="cuda", generator=gen).bfloat16()
    ids = torch.randint(0, V, (some, k), device="cuda", generator=gen, dtype=torch.int32)
    values, w = torch.randn((some, k), device="cuda", generator=gen), torch.randn(some, device="cuda", generator=gen)
    one = distill_loss(z, ids, values, w, temperature=2.0, gradient=True)
    at = torch.arange(T, device="cuda") % some
    given = ids[at].contiguous(), values[at].contiguous()
    d = distill_loss(z[at], *given, w[at], temperature=2.0, gradient=True)
    assert torch.equal(d.loss, one.loss[at]) and torch.equal(d.Z, one.Z[at]) and torch.equal(d.m, one.m[at])
    step = 7 << 15
    assert all(torch.equal(d.dlogits[a:a + step], one.dlogits[at[a:a + step]]) for a in range(0, T, step))
    d.dlogits = None
    back = distill_backward(z[at], d.m, d.Z, *given, w[at], temperature=2.0)
    assert all(torch.equal(back[a:a + step], one.dlogits[at[a:a + step]]) for a in range(0, T, step))


@pytest.mark.parametrize("T,width,gated", [((1 << 22) + 5, 16, False), ((1 << 22) + 5, 32, True), ((1 << 20) + 3, 2064, False)])
def test_quantised_rows(T, width, gated):
    torch = require_gpu()
    from paper_2609_36301_amd import quantize_rows
    announce("quantize_rows T=%d width=%d gated=%s" % (T, width, gated))
    gen = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn((7, width * (2 if gated else 1)), device="cuda", generator=gen).bfloat16()
    one = quantize_rows(x, gated=gated)
    at = torch.arange(T, device="cuda") % 7
    many = quantize_rows(x[at], gated=gated)
    assert torch.equal(many.scale, one.scale[at])
    step = 7 << 15
    assert all(torch.equal(many.q[a:a + step], one.q[at[a:a + step]]) for a in range(0, T, step))


@pytest.mark.parametrize("k", [1, 2])
def test_linear_maps(k):
    """More tiles and more experts than workgroups (2^19)."""
    torch = require_gpu()
    from paper_2609_36301_amd import dispatch_sort, expert_linear, expert_linear_backward, expert_linear_q8
    T, K, N, M = 400000, 16, 16, 700000
    announce("expert_linear T=%d K=%d N=%d M=%d k=%d" % (T, K, N, M, k))
    gen = torch.Generator(device="cuda").manual_seed(7)
    normal = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)  # noqa: E731
    x, W, dy = normal(T, K), normal(M, N, K), normal(T * k, N)
    idx = torch.randint(0, M + 20000, (T, k), device="cuda", generator=gen, dtype=torch.int32)
    sel = (idx, *dispatch_sort(idx, M))
    e = idx.flatten().long()
    there = (e < M)[:, None]
    rows = torch.arange(T, device="cuda").repeat_interleave(k)
    We = W[e.clamp(max=M - 1)].double() * there[:, :, None]
    xe, de = x.double()[rows], dy.double() * there

    def within(got, want, size, terms):
        """`terms` fp32 additions of terms whose magnitudes add up to `size`, one rounding to bf16"""
        bound = terms * E32 * size * (1 + E16) + E16 * want.abs() + 1e-37
        worst = ((got.double() - want).abs() / bound).max().item()
        assert worst <= 1, "%.3g times the bound off" % worst

    y = expert_linear(x, W, *sel)
    within(y, (We * xe[:, None]).sum(2), (We * xe[:, None]).abs().sum(2), K)
    assert not y[e >= M].any()
    g = expert_linear_backward(x, W, *sel, dy)
    shares = (We * de[:, :, None])
    within(g.dx, shares.sum(1).view(T, k, K).sum(1), shares.abs().sum(1).view(T, k, K).sum(1), N + k)
    del shares
    outer = de[:, :, None] * xe[:, None]
    dW, size = (torch.zeros((M + 1, N, K), dtype=torch.float64, device="cuda") for _ in range(2))
    dW.index_add_(0, e.clamp(max=M), outer)
    size.index_add_(0, e.clamp(max=M), outer.abs())
    # (a full expert here has at most 64 entries)
    assert torch.bincount(e, minlength=M)[:M].max() <= 64
    within(g.dWt, dW[:M], size[:M], 64)
    del outer, dW, size
    q = torch.randint(-128, 128, (T, K), device="cuda", generator=gen, dtype=torch.int8)
    Wq = torch.randint(-128, 128, (M, N, K), device="cuda", generator=gen, dtype=torch.int8)
    out = expert_linear_q8(q, torch.ones(T, device="cuda"), Wq, torch.ones((M, N), device="cuda"), *sel, out_dtype=torch.float32)
    want = (Wq[e.clamp(max=M - 1)].double() * q.double()[rows][:, None]).sum(2) * there
    assert torch.equal(out.double(), want)  # (whole numbers below 2^24)
