"""Distillation on rows of millions of classes: the sum of the exponentials against 64 bits."""
import pytest

from gpu_util import announce, require_gpu

pytestmark = pytest.mark.gpu

E32 = 2.0 ** -24
HALF = {32: E32, 16: 2.0 ** -8}


def rows(V, bits, kind):
    """Two rows: nearly constant (where a running sum's roundings all go one way) or ascending (where its maximum moves
    with every step), and a largest class."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(V)
    if kind == "constant":
        z = torch.full((2, V), -0.3, device="cuda")
        z[1] += 0.01 * torch.randn(V, device="cuda", generator=gen)
    else:
        z = torch.linspace(-2.0, 0.0, V, device="cuda", dtype=torch.float64).float().repeat(2, 1)
        z[1] *= 15.0
    z[:, V // 3] = 0.5
    return z if bits == 32 else z.bfloat16()


@pytest.mark.parametrize("bits", [16, 32])
@pytest.mark.parametrize("kind", ["constant", "ascending"])
@pytest.mark.parametrize("V", [(1 << 20) + 1, (1 << 22) + 3, (1 << 26) + 5])
def test_sums_of_long_rows(V, kind, bits):
    """Z is a sum of positive terms: a thread adds at most 64 of them one after the other, and these sums join in two floats.
    Their base moves when the maximum has grown by 2^8, so that three moves at most count (at 2^17 terms a thread), each a
    factor of 4 E32 and 3 E32 times an exponent of 8 ln 2; 22 steps join the threads: 64 + 60 + 22 + 2 roundings, and those of
    an exponential (4 E32 and 3 E32 times its exponent, at most 31 here) in its terms."""
    torch = require_gpu()
    from paper_2609_36301_amd import distill_backward, distill_loss
    z = rows(V, bits, kind)
    k, tau = 3, 1.0
    ids = torch.tensor([[V // 3, 5, V - 1]] * 2, dtype=torch.int32, device="cuda")
    values = torch.tensor([[2.0, 1.0, 0.0]] * 2, device="cuda")
    weight = torch.tensor([1.0, float(V)], device="cuda")
    x = (z.double() - 0.5) / tau
    e = x.exp()
    Z = e.sum(1)
    spread = (e * x.abs()).sum(1) / Z
    del x
    rel = (64 + 60 + 22 + 2 + 4 + 3 * spread) * E32
    q = torch.softmax(values.double() / tau, 1)
    at = torch.gather(z.double(), 1, ids.long())
    loss = tau * tau * (q * (q.log() - (at - 0.5) / tau + Z.log()[:, None])).sum(1)
    # the logarithm's relative error, and the roundings of the other terms (below 64 in sum)
    bound = tau * tau * (rel + 64 * E32 * (1 + Z.log()))
    want = e / Z[:, None]
    slack = want * (rel[:, None] + (16 + 3 * 31) * E32)
    want.scatter_add_(1, ids.long(), -q)
    slack.scatter_add_(1, ids.long(), 64 * E32 * q)
    want *= weight.double()[:, None] * tau
    slack *= weight.double()[:, None] * tau
    slack += HALF[bits] * want.abs() + 1e-37
    del e
    announce("distill V=%d bits=%d %s, the loss alone" % (V, bits, kind))
    alone = distill_loss(z, ids, values, temperature=tau)
    announce("distill V=%d bits=%d %s, loss and gradient" % (V, bits, kind))
    both = distill_loss(z, ids, values, weight, temperature=tau, gradient=True)
    announce("distill V=%d bits=%d %s, backward" % (V, bits, kind))
    back = distill_backward(z, alone.m, alone.Z, ids, values, weight, temperature=tau)
    for d, what in ((alone, "the loss alone"), (both, "loss and gradient")):
        off = ((d.Z.double() - Z).abs() / Z / rel).max().item()
        assert off <= 1, "%s: Z is %.3g times its bound off" % (what, off)
        assert (d.m == 0.5).all()
        off = ((d.loss.double() - loss).abs() / bound).max().item()
        assert off <= 1, "%s: the loss is %.3g times its bound off" % (what, off)
    for grad, what in ((both.dlogits, "loss and gradient"), (back, "backward")):
        off = ((grad.double() - want).abs() / slack).max().item()
        assert off <= 1, "%s: the gradient is %.3g times its bound off" % (what, off)
