"""The 64-bit forms of the linear maps and of the distillation loss against differences (CPU)."""
import numpy as np
import pytest

import linear_ref as ref


def test_linear_gradients_are_differences():
    rng = np.random.default_rng(1)
    T, K, N, M, k = 5, 8, 8, 3, 2
    x, W = rng.standard_normal((T, K)), rng.standard_normal((M, N, K))
    idx, c = rng.integers(-1, M + 1, (T, k)), rng.standard_normal((T * k, N))
    f = lambda x, W: float((ref.linear(x, W, idx)[0] * c).sum())  # noqa: E731
    (dx, dW), _ = ref.linear_backward(x, W, idx, c)
    for grad, at in ((dx, x), (dW, W)):
        for i in rng.integers(0, at.size, 12):
            v, step = at.ravel()[i], 1e-4
            at.ravel()[i] = v + step
            up = f(x, W)
            at.ravel()[i] = v - step
            down = f(x, W)
            at.ravel()[i] = v
            assert abs((up - down) / (2 * step) - grad.ravel()[i]) < 1e-7 * (1 + abs(grad.ravel()[i]))


@pytest.mark.parametrize("tau", [0.5, 1.0, 3.0])
def test_distill_gradient_is_differences(tau):
    rng = np.random.default_rng(2)
    T, V, k = 4, 11, 5
    z, v = rng.standard_normal((T, V)), rng.standard_normal((T, k))
    ids = rng.integers(0, V, (T, k))  # (an id may occur twice)
    ids[1, 2], ids[3] = -1, V
    v[2, 0] = -np.inf
    w = rng.random(T)
    (loss, _, _, grad), _ = ref.distill(z, ids, v, tau, w)
    assert loss[3] == 0 and not grad[3].any() and (loss[:3] != 0).all()
    for t in range(T):
        for e in range(V):
            two = []
            for step in (1e-4, -1e-4):
                y = z.copy()
                y[t, e] += step
                two.append((ref.distill(y, ids, v, tau)[0][0] * w).sum())
            assert abs((two[0] - two[1]) / 2e-4 - grad[t, e]) < 1e-6


def test_quantize_ties_and_special_rows():
    x = np.zeros((6, 16))
    x[0, :3] = [2.0, 1.0, -1.0]      # 63.5: to even
    x[1, 0] = 2.0 ** -101
    x[2, 0], x[3, 0] = np.inf, np.nan
    x[4] = -1.0
    q, scale = ref.quantize(x)
    assert q[0, :3].tolist() == [127, 64, -64] and scale[0] == np.float32(2.0 / 127)
    assert not q[1].any() and scale[1] == 0 and not q[5].any() and scale[5] == 0
    assert np.isnan(scale[2:4]).all() and not q[2:4].any() and (q[4] == -127).all()
