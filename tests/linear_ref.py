"""The experts' linear maps, the quantisation of rows and the distillation loss in 64 bits (numpy), and how far a
result may be from each.

As in layer_ref: a rounding is off by at most half a step (E16, E32 relative to the value), a sum of n fp32 terms by
at most n E32 times the sum of their magnitudes.
"""
from __future__ import annotations

import numpy as np

from layer_ref import E16, E32, TINY, experts

ROW_TINY = 2.0 ** -100


def _half(bits):
    return E32 if bits == 32 else E16


def linear(x, Wt, idx, bits=16):
    """y [T k][N] and its bound: K exact products summed in fp32, one rounding."""
    T, k = idx.shape
    M, N, K = Wt.shape
    y, mag = np.zeros((T * k, N)), np.zeros((T * k, N))
    for e, p in experts(idx, M):
        y[p] = x[p // k] @ Wt[e].T
        mag[p] = np.abs(x[p // k]) @ np.abs(Wt[e].T)
    return y, K * E32 * mag * (1 + E16) + _half(bits) * np.abs(y) + TINY


def linear_backward(x, Wt, idx, dy):
    """(dx, dW) and the bound of each: sums of N products per entry and k entries, or of an expert's entries."""
    T, k = idx.shape
    M, N, K = Wt.shape
    dx, mx = np.zeros((T, K)), np.zeros((T, K))
    dW, bW = np.zeros((M, N, K)), np.full((M, N, K), TINY)
    for e, p in experts(idx, M):
        t = p // k
        np.add.at(dx, t, dy[p] @ Wt[e])
        np.add.at(mx, t, np.abs(dy[p]) @ np.abs(Wt[e]))
        dW[e] = dy[p].T @ x[t]
        bW[e] += (len(p) + 33) * E32 * (np.abs(dy[p]).T @ np.abs(x[t])) * (1 + E16) + E16 * np.abs(dW[e])
    return (dx, dW), ((N + k) * E32 * mx * (1 + E16) + E16 * np.abs(dx) + TINY, bW)


def quantize(x):
    """q and scale of rows of float64 values, to the bit where the values are bf16: the inverse is rounded to fp32 (a
    quotient of numbers of at most 24 bits is never nearer to a border of fp32 than fp64 tells), its product with a
    value has at most 48 bits."""
    with np.errstate(all="ignore"):
        a = np.abs(x).max(axis=1)
        bad = ~np.isfinite(x).all(axis=1)
        live = (a >= ROW_TINY) & ~bad
        inv = np.where(live, (127.0 / a).astype(np.float32).astype(np.float64), 0.0)
        q = np.where(live[:, None], np.rint(np.where(live[:, None], x, 0.0) * inv[:, None]), 0.0)
        scale = np.where(bad, np.nan, np.where(live, a / 127.0, 0.0)).astype(np.float32)
    return q.astype(np.int8), scale


def gated(x):
    """silu(g) u of rows [g u], and how far fp32 may be from it: sigma comes from exp2 and reciprocal."""
    g, u = np.split(x, 2, axis=1)
    v = g / (1.0 + np.exp(-g)) * u
    return v, (12 + np.abs(g)) * E32 * np.abs(v) + TINY


def linear_q8(q, q_scale, Wq, w_scale, idx, gate=None, bits=16):
    """y [T k][N] and its bound: the exact sum, its conversion to fp32, three products, one rounding."""
    T, k = idx.shape
    M, N, K = Wq.shape
    y = np.zeros((T * k, N))
    for e, p in experts(idx, M):
        acc = q[p // k].astype(np.float64) @ Wq[e].astype(np.float64).T  # (exact: below 2^53)
        g = 1.0 if gate is None else gate.ravel()[p][:, None]
        y[p] = acc * w_scale[e] * (q_scale[p // k][:, None] * g)
    return y, (4 * E32 + _half(bits)) * np.abs(y) * (1 + E16) + TINY


def distill(z, ids, values, tau, weight=None, bits=16):
    """loss, m, Z and the weighted gradient [T][V], and the bounds of loss, Z and gradient.

    A thread adds at most 128 exponentials one after the other and at most 26 such sums meet (5 steps more for rows
    that are read twice): 200 E32 of a sum of positive numbers; an exponential is off by 4 E32 and by 3 E32 times its
    exponent (difference, factor, product); a logarithm of at most 2^30 by 64 E32."""
    T, V = z.shape
    w = np.ones(T) if weight is None else weight
    with np.errstate(all="ignore"):
        m = z.max(axis=1)
        x = (z - m[:, None]) / tau
        e = np.exp(x)
        Z = e.sum(axis=1)
        P = e / Z[:, None]
        ax = np.where(np.isfinite(x), np.abs(x), 0.0)
        spread = (P * ax).sum(axis=1)  # mean exponent: what its errors make of the sum
    eZ = (200 + 4 + 3 * spread) * E32 * Z
    valid = (ids >= 0) & (ids < V) & (values != -np.inf)
    loss, grad = np.zeros(T), np.zeros((T, V))
    bl, bg = np.full(T, TINY), np.full((T, V), TINY)
    k = ids.shape[1]
    for t in range(T):
        j = np.flatnonzero(valid[t])
        if len(j) == 0:
            continue
        d = values[t, j] - values[t, j].max()
        u = np.exp(d / tau)
        U = u.sum()
        q = u / U
        some = q > 0
        rel = (k + 12 + 6 * np.abs(d) / tau) * E32  # of q
        D = np.where(some, d - (z[t, ids[t, j]] - m[t]), 0.0)
        Dmag = np.where(some, np.abs(d) + np.abs(z[t, ids[t, j]] - m[t]), 0.0)
        loss[t] = tau * tau * (np.log(Z[t]) - np.log(U) + (q * D).sum() / tau)
        bl[t] += tau * tau * (eZ[t] / Z[t] + (k + 8) * E32 + 128 * E32 + (q * Dmag * (rel + (k + 8) * E32)).sum() / tau)
        bl[t] += 8 * E32 * tau * tau * (abs(np.log(Z[t])) + abs(np.log(U)) + (q * Dmag).sum() / tau)
        Q, eQ = np.zeros(V), np.zeros(V)
        np.add.at(Q, ids[t, j], q)
        np.add.at(eQ, ids[t, j], q * (rel + (k + 8) * E32))
        grad[t] = w[t] * tau * (P[t] - Q)
        eP = P[t] * (eZ[t] / Z[t] + (12 + 3 * ax[t]) * E32)
        bg[t] += abs(w[t]) * tau * (eP + eQ + 4 * E32 * (P[t] + Q)) * (1 + E16) + _half(bits) * np.abs(grad[t])
    return (loss, m, Z, grad), (bl, eZ, bg)
