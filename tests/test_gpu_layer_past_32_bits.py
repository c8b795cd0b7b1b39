"""The layer's calls on single tensors and experts of more than 2^31 elements (marked `gpu`)."""
import numpy as np
import pytest

import layer_ref as ref
from gpu_util import announce, require_gpu
from test_gpu_ffn import check

pytestmark = pytest.mark.gpu


def test_an_expert_of_the_largest_size():
    """h = s = 65536, 12.9 G weights in one expert: all zero but for the rows of a few hidden units over the whole range,
    so that the result is that of an expert of these units alone (sums with zeros are exact), and every other gradient
    is zero."""
    torch = require_gpu()
    from paper_2609_36301_amd import layer
    T, h, s = 3, 65536, 65536
    units = [0, 5, 63, 64, 16383, 16384, 32768, 49151, 65528, 65535]
    rows = torch.tensor(units + [s + u for u in units], device="cuda")
    cols = torch.tensor(units, device="cuda")
    announce("expert_ffn and its backward pass, one expert of h = s = 65536")
    gen = torch.Generator(device="cuda").manual_seed(5)
    normal = lambda *n, scale=1.0: torch.empty(n, dtype=torch.bfloat16, device="cuda").normal_(0, scale, generator=gen)  # noqa: E731
    x, du, gate = normal(T, h), normal(T, h, scale=0.1), torch.rand((T, 1), device="cuda", generator=gen)
    W1, W2 = torch.zeros((1, 2 * s, h), dtype=torch.bfloat16, device="cuda"), torch.zeros(
        (1, h, s), dtype=torch.bfloat16, device="cuda")
    w1, w2 = normal(len(rows), h, scale=h ** -0.5), normal(h, len(cols), scale=0.3)
    W1[0, rows], W2[0, :, cols] = w1, w2
    idx = torch.zeros((T, 1), dtype=torch.int32, device="cuda")
    offsets, srt = torch.tensor([0, T], dtype=torch.int32, device="cuda"), torch.arange(T, dtype=torch.int32, device="cuda")
    y = layer.expert_ffn(x, W1, W2, idx, offsets, srt, gate)
    got = layer.expert_ffn_backward(x, W1, W2, idx, offsets, srt, gate, du)
    torch.cuda.synchronize()
    e = lambda t: t.double().cpu().numpy()  # noqa: E731
    given = (e(x), e(w1)[None], e(w2)[None], idx.cpu().numpy(), e(gate))
    want, bound = ref.ffn(*given)
    check("y", y.float().cpu().numpy(), want, bound, "largest expert")
    want, bound = ref.ffn_backward(*given, e(du))
    small = (got.dx, got.dW1t[:, rows], got.dW2t[:, :, cols], got.dgate)
    for name, g, v, b in zip(("dx", "dW1t", "dW2t", "dgate"), small, want, bound):
        check(name, g.float().cpu().numpy(), v, b, "largest expert")
    got.dW1t[:, rows], got.dW2t[:, :, cols] = 0, 0
    for t in (got.dW1t[0], got.dW2t[0]):
        for a in range(0, t.shape[0], 8192):
            assert not t[a:a + 8192].any()


def test_norms():
    torch = require_gpu()
    from paper_2609_36301_amd import layer
    T, h, eps = (1 << 19) + 9, 4112, 1e-5
    assert T * h > 2 ** 31
    announce("block_norm and its backward pass T=%d h=%d" % (T, h))
    gen = torch.Generator(device="cuda").manual_seed(6)
    normal = lambda: torch.empty((T, h), dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=gen)  # noqa: E731
    r, y, dxn = normal(), normal(), normal()
    w, gate = torch.rand(h, device="cuda") + 0.5, torch.rand(T, device="cuda")
    out = layer.block_norm(r, y, w_after=w, w_before=w, gate=gate, eps=eps, save_u=True)
    back = layer.block_norm_backward(out.u, out.r, r, dxn, w_after=w, w_before=w, gate=gate, eps=eps)
    torch.cuda.synchronize()
    wd, e32 = w.double().cpu().numpy(), np.float32(eps).item()
    for rows in (slice(0, 2), slice((1 << 31) // h - 1, (1 << 31) // h + 2), slice(T - 3, T)):
        e = lambda t: t[rows].double().cpu().numpy()  # noqa: E731
        want, bound = ref.block_norm(e(r), e(y)[:, None], wd, wd, e(gate), 1.0, e32, True, 16)
        for name, v, b in zip(("r", "xn", "u"), want, bound):
            check(name, getattr(out, name)[rows].float().cpu().numpy(), v, b, str(rows))
        want, bound = ref.block_norm_backward(e(out.u), e(out.r), e(r), e(dxn), wd, wd, e(gate), 1.0, e32, True, 16)
        for name in ("dr", "du", "dgate"):
            i = ("dr", "du", "dw_after", "dw_before", "dgate").index(name)
            check(name, getattr(back, name)[rows].float().cpu().numpy(), want[i], bound[i], str(rows))


def test_clipping():
    """Powers of two, whose squares add up exactly in fp64."""
    torch = require_gpu()
    from paper_2609_36301_amd import layer
    n = (1 << 31) + 4099
    announce("clip tensors of %d elements" % n)
    a = torch.full((n,), 2.0 ** -10, dtype=torch.bfloat16, device="cuda")
    b = torch.full((n,), -2.0 ** -12, device="cuda")
    a[-2], b[-1] = 64.0, 32.0
    norm = ((n - 1) * 2.0 ** -20 + 2.0 ** 12 + (n - 1) * 2.0 ** -24 + 2.0 ** 10) ** 0.5
    got = layer.clip_gradients([a, b], norm / 2)
    torch.cuda.synchronize()
    assert abs(float(got) / norm - 1) <= 2.0 ** -24 + 1e-12
    for t, v, last, at in ((a, 2.0 ** -10, 64.0, n - 2), (b, -2.0 ** -12, 32.0, n - 1)):
        step = ref.E16 if t.dtype == torch.bfloat16 else ref.E32
        tol = lambda w: (step + 2.1 * ref.E32 + 1e-6 / norm) * abs(w)  # noqa: E731
        assert abs(float(t[at]) - last / 2) <= tol(last / 2)
        t[at] = v / 2
        for c in range(0, n, 1 << 29):
            piece = t[c:c + (1 << 29)]
            assert abs(float(piece.max()) - v / 2) <= tol(v / 2) and abs(float(piece.min()) - v / 2) <= tol(v / 2)
