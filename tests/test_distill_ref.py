"""The 60-digit form of the distillation loss against the 64-bit one, and that its bounds are small beside what they bound
(CPU)."""
import numpy as np
import pytest

import distill_ref
import linear_ref


def rows(seed, T, V, k):
    rng = np.random.default_rng(seed)
    z, v = rng.standard_normal((T, V)).astype(np.float32), rng.standard_normal((T, k)).astype(np.float32)
    ids = np.stack([rng.permutation(V)[:k] for _ in range(T)]) if k <= V else rng.integers(0, V, (T, k))
    return z.astype(np.float64), ids, v.astype(np.float64), rng.random(T)


@pytest.mark.parametrize("V,k", [(1, 1), (7, 7), (11, 6), (11, 17), (64, 64)])
@pytest.mark.parametrize("tau", [0.25, 1.0, 20.0])
def test_both_forms(V, k, tau):
    z, ids, v, w = rows(V + k, 3, V, k)
    if V > 1:
        z[1, 0], v[2, 0], ids[0, 1] = -np.inf, -np.inf, -1
        ids[1][ids[1] == 0] = 1
    (loss, grad), (bl, bg) = distill_ref.distill(z, ids, v, tau, w)
    (want, _, _, wgrad), _ = linear_ref.distill(z, ids, v, tau, w)
    assert np.abs(loss - want).max() < 1e-13 * tau * tau * (1 + np.log(V + k)) * 10
    assert np.abs(grad - wgrad).max() < 1e-13 * tau
    assert np.isfinite(bl).all() and np.isfinite(bg).all() and (bl > 0).all()


@pytest.mark.parametrize("tau", [1.0, 20.0, 256.0, 4096.0, 2.0 ** 20, 2.0 ** 40])
def test_bounds_are_relative(tau):
    """Where the entries cover all classes: a thousandth of the loss, and of the gradient's largest entries, at every
    temperature."""
    z, ids, v, _ = rows(5, 4, 64, 64)
    (loss, grad), (bl, bg) = distill_ref.distill(z, ids, v, tau)
    assert (loss > 0.1).all() and (bl < 1e-3 * loss).all()
    assert (bg.max(1) < 1e-3 * np.abs(grad).max(1)).all()
