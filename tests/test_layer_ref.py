"""The 64-bit reference of the layer's operators on the CPU: its gradients against central differences of
its forward passes, and the Sort + Count it uses against the oracle's."""
import numpy as np
import pytest

import layer_ref as ref
import oracle


def _difference(f, v, w, step=1e-5):
    """Directional derivative of sum(f * w) along a random direction: (numeric, direction)."""
    d = np.random.default_rng(3).standard_normal(v.shape)
    return ((f(v + step * d) * w).sum() - (f(v - step * d) * w).sum()) / (2 * step), d


@pytest.mark.parametrize("gated", [True, False])
def test_ffn_gradients_are_those_of_the_forward_pass(gated):
    rng = np.random.default_rng(0)
    T, h, s, M, k = 7, 16, 8, 4, 3
    idx = rng.integers(-1, M + 1, size=(T, k)).astype(np.int32)
    idx[2] = idx[2, 0]  # one id several times in a token
    x, W1, W2 = rng.standard_normal((T, h)), rng.standard_normal((M, 2 * s, h)), rng.standard_normal((M, h, s))
    gate = rng.random((T, k)) if gated else None
    du = rng.standard_normal((T, h))
    total = lambda *a: ref.ffn(*a)[0].reshape(T, k, h).sum(1)  # noqa: E731
    (dx, dW1, dW2, dgate), _ = ref.ffn_backward(x, W1, W2, idx, gate, du)
    cases = [(lambda v: total(v, W1, W2, idx, gate), x, dx), (lambda v: total(x, v, W2, idx, gate), W1, dW1),
             (lambda v: total(x, W1, v, idx, gate), W2, dW2)]
    if gated:
        cases.append((lambda v: total(x, W1, W2, idx, v), gate, dgate))
    for f, at, grad in cases:
        want, d = _difference(f, at, du)
        assert abs((grad * d).sum() - want) <= 1e-6 * (np.abs(grad * d).sum() + 1)


@pytest.mark.parametrize("norm_after,gated,block", [(True, True, True), (False, True, True), (True, False, True),
                                                    (True, False, False)])
def test_norm_gradients_are_those_of_the_forward_pass(norm_after, gated, block):
    rng = np.random.default_rng(1)
    T, h, eps, alpha = 5, 16, 1e-3, 0.7
    r, u = rng.standard_normal((T, h)), rng.standard_normal((T, h))
    wa, wb = (rng.standard_normal(h) if block else None), rng.standard_normal(h)
    gate = rng.random(T) if gated else None
    a = alpha if block else 1.0
    c_r, c_x = rng.standard_normal((T, h)), rng.standard_normal((T, h))

    def run(r, u, wa, wb, gate):
        y = u[:, None] if block else None
        (r1, xn, _), _ = ref.block_norm(r, y, wa, wb, gate, a, eps, norm_after, 32)
        return np.concatenate([r1, xn])

    r_out = run(r, u, wa, wb, gate)[:T]
    grads, _ = ref.block_norm_backward(u if block else None, r_out, c_r, c_x, wa, wb, gate, a, eps, norm_after, 32)
    cot = np.concatenate([c_r, c_x])
    args = [r, u, wa, wb, gate]
    for i, g in ((0, grads[0]), (1, grads[1]), (2, grads[2]), (3, grads[3]), (4, grads[4])):
        if g is None or args[i] is None:
            continue
        want, d = _difference(lambda v: run(*(args[:i] + [v] + args[i + 1:])), args[i], cot)
        assert abs((g * d).sum() - want) <= 1e-6 * (np.abs(g * d).sum() + 1), i


@pytest.mark.parametrize("T,k,M", [(1, 1, 1), (5, 3, 4), (100, 2, 7), (3, 32, 1000)])
def test_dispatch_is_the_oracles(T, k, M):
    idx = np.random.default_rng(T).integers(-1, M + 1, size=(T, k)).astype(np.int32)
    offsets, srt = ref.dispatch(idx, M)
    want_o, want_s = oracle.dispatch_sort(idx, M)
    assert np.array_equal(offsets, want_o) and np.array_equal(srt, want_s)
