"""The linear maps, quantised rows and distillation where an operand or a result has more than 2^31 elements (marked `gpu`).
Random rows and columns are compared with their 64-bit forms."""
import numpy as np
import pytest

import linear_ref as ref
from gpu_util import announce, require_gpu

pytestmark = pytest.mark.gpu
MOST = 2 ** 31


def normal(gen, *shape, scale=1.0):
    import torch
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0, scale, generator=gen)


def one_map(T):
    """idx, offsets and sorted of one dense map."""
    import torch
    i32 = {"dtype": torch.int32, "device": "cuda"}
    return torch.zeros((T, 1), **i32), torch.tensor([0, T], **i32), torch.arange(T, **i32)


def np64(t):
    return t.double().cpu().numpy()


def within(got, want, bound):
    assert np.max(np.abs(got - want) / bound) <= 1.0


def test_many_rows():
    """x, y and dy of more than 2^31 elements, and dx."""
    torch = require_gpu()
    from paper_2609_36301_amd import expert_linear, expert_linear_backward
    T, K, N = 1 << 20, 2056, 2064
    assert T * K > MOST and T * N > MOST
    announce("expert_linear T=%d K=%d N=%d" % (T, K, N))
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, W, sel = normal(gen, T, K), normal(gen, 1, N, K, scale=K ** -0.5), one_map(T)
    y = expert_linear(x, W, *sel)
    rows = torch.tensor([0, 1, 255, T // 2, T - 2, T - 1], device="cuda")
    zero = np.zeros((len(rows), 1), np.int32)
    within(np64(y[rows]), *ref.linear(np64(x[rows]), np64(W), zero))
    dy = y
    g = expert_linear_backward(x, W, *sel, dy, need_dW=False)
    (dx, _), (bound, _) = ref.linear_backward(np64(x[rows]), np64(W), zero, np64(dy[rows]))
    within(np64(g.dx[rows]), dx, bound)


def test_large_weights():
    """W and dW of more than 2^31 elements, in bf16 and in 8 bits."""
    torch = require_gpu()
    from paper_2609_36301_amd import dispatch_sort, expert_linear, expert_linear_backward, expert_linear_q8, quantize_rows
    T, K, N, M, k = 6000, 1040, 1040, 2000, 1
    assert M * N * K > MOST
    announce("expert_linear T=%d K=%d N=%d M=%d" % (T, K, N, M))
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, W = normal(gen, T, K), normal(gen, M, N, K, scale=K ** -0.5)
    idx = torch.randint(0, M, (T, k), device="cuda", generator=gen, dtype=torch.int32)
    idx[-3:] = M - 1
    sel = (idx, *dispatch_sort(idx, M))
    y = expert_linear(x, W, *sel)
    dy = normal(gen, T, N)
    g = expert_linear_backward(x, W, *sel, dy)
    xq, Wq = quantize_rows(x), quantize_rows(W)
    yq = expert_linear_q8(xq.q, xq.scale, Wq.q, Wq.scale, *sel)
    for e in (0, M // 2, int(idx[0, 0]), M - 1):
        t = (idx[:, 0] == e).nonzero()[:, 0]
        zero = np.zeros((len(t), 1), np.int32)
        We = np64(W[e:e + 1])
        (dx, dW), (bx, bW) = ref.linear_backward(np64(x[t]), We, zero, np64(dy[t]))
        within(np64(g.dWt[e]), dW[0], bW[0])
        if len(t):
            within(np64(y[t]), *ref.linear(np64(x[t]), We, zero))
            within(np64(g.dx[t]), dx, bx)
            q, scale = ref.quantize(We[0])
            assert np.array_equal(Wq.q[e].cpu().numpy(), q) and np.array_equal(Wq.scale[e].cpu().numpy(), scale)
            within(np64(yq[t]), *ref.linear_q8(xq.q[t].cpu().numpy(), np64(xq.scale[t]), q[None], scale[None].astype(np.float64), zero))


@pytest.mark.parametrize("bits", [16, 32])
def test_many_logits(bits):
    torch = require_gpu()
    from paper_2609_36301_amd import distill_backward, distill_loss
    T, V, k = 70000, 32001, 6
    assert T * V > MOST
    announce("distill T=%d V=%d bits=%d" % (T, V, bits))
    gen = torch.Generator(device="cuda").manual_seed(3)
    z = normal(gen, T, V, scale=2.0)
    z = z.float() if bits == 32 else z
    ids = torch.randint(0, V, (T, k), device="cuda", generator=gen, dtype=torch.int32)
    values, w = torch.randn((T, k), device="cuda", generator=gen), torch.rand(T, device="cuda", generator=gen)
    rows = torch.tensor([0, 1, T // 2, T - 1], device="cuda")
    d = distill_loss(z, ids, values, w, temperature=2.0, gradient=True)
    (loss, m, Z, grad), (bl, bZ, bg) = ref.distill(np64(z[rows]), ids[rows].cpu().numpy(), np64(values[rows]), 2.0, np64(w[rows]), bits)
    within(np64(d.loss[rows]), loss, bl)
    within(np64(d.dlogits[rows]), grad, bg)
    first = d.dlogits[rows].clone()
    del d.dlogits
    two = distill_backward(z, d.m, d.Z, ids, values, w, temperature=2.0)
    assert torch.equal(two[rows], first)
