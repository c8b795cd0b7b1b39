"""The layer around the router in 64 bits (numpy), and how far a result may be from it.

Every function takes float64 arrays (exact values of the bf16 or fp32 inputs).  The bounds follow the
kernels' stated numerics: bf16 operands with fp32 accumulation, one rounding to bf16 where it is stated.
A rounding is off by at most half a step: E16 = 2^-8 (bf16), E32 = 2^-24 (fp32) relative to the value;
a sum of n fp32 terms is off by at most n E32 times the sum of their magnitudes.
"""
from __future__ import annotations

import numpy as np

E16, E32 = 2.0 ** -8, 2.0 ** -24
TINY = 1e-30  # below any value used here: roundings of results near zero


def to_bf16(a):
    """float64/float32 -> bf16 bit patterns (round to nearest even) as uint16."""
    from paper_2609_36301_amd.inputs import f32_to_bf16_bits
    return f32_to_bf16_bits(np.asarray(a, dtype=np.float32))


def from_bf16(b):
    from paper_2609_36301_amd.inputs import bf16_bits_to_f32
    return bf16_bits_to_f32(b).astype(np.float64)


def dispatch(idx, M):
    """offsets [M + 1] and sorted [T k] of Sort + Count."""
    flat = idx.ravel().astype(np.int64)
    key = np.where((flat >= 0) & (flat < M), flat, M)
    srt = np.argsort(key, kind="stable").astype(np.int32)
    return np.searchsorted(key[srt], np.arange(M + 1), side="left").astype(np.int32), srt


def _hidden(X, W1, s):
    """G, U, sigma, silu, A and their bounds (errors of G, U and A before its rounding)."""
    h = X.shape[1]
    gu, mag = X @ W1.T, np.abs(X) @ np.abs(W1.T)
    G, U = gu[:, :s], gu[:, s:]
    eG, eU = (h + 2) * E32 * mag[:, :s], (h + 2) * E32 * mag[:, s:]
    sig = 1.0 / (1.0 + np.exp(-G))
    silu = G * sig
    A = silu * U
    # sigma comes from exp2 and reciprocal: a few steps, and |G| E32 in the exponent; |silu'| <= 1.1
    e_sig = (8 + np.abs(G)) * E32 * sig
    eA = 1.1 * eG * np.abs(U) + np.abs(silu) * eU + (np.abs(G) * e_sig + 4 * E32 * np.abs(silu)) * np.abs(U)
    return G, U, sig, silu, A, eG, eU, e_sig, eA


def experts(idx, M):
    """(expert, flat entries of it) for the experts that some entry selects."""
    flat = idx.ravel()
    for e in np.unique(flat):
        if 0 <= e < M:
            yield int(e), np.flatnonzero(flat == e)


def ffn(x, W1t, W2t, idx, gate, planes=1):
    """y [T k][h] and its bound; planes: the bf16 addends that A is rounded to (the second one takes what the
    first leaves, at most E16 of it, and is off by E16 of that)."""
    kept = E16 ** planes
    T, k = idx.shape
    M, h, s = W2t.shape
    g = np.ones(T * k) if gate is None else gate.ravel()
    y, bound = np.zeros((T * k, h)), np.zeros((T * k, h))
    for e, p in experts(idx, M):
        A, eA = (lambda r: (r[4], r[8]))(_hidden(x[p // k], W1t[e], s))
        W2 = W2t[e].T
        c = g[p][:, None]
        y[p] = c * (A @ W2)
        mag = np.abs(c) * (np.abs(A) @ np.abs(W2))
        bound[p] = (np.abs(c) * ((eA + kept * (np.abs(A) + eA)) @ np.abs(W2)) * (1 + 2 * E16)
                    + (planes * s + 4) * E32 * mag + E16 * np.abs(y[p]) * (1 + 2 * E16) + TINY)
    return y, bound


def ffn_backward(x, W1t, W2t, idx, gate, du, planes=1):
    """(dx, dW1t, dW2t, dgate) and the bound of each; planes as for ffn, of [dG dU] and gate A."""
    kept = E16 ** planes
    T, k = idx.shape
    M, h, s = W2t.shape
    g = np.ones(T * k) if gate is None else gate.ravel()
    dx, dW1, dW2, dg = np.zeros((T, h)), np.zeros((M, 2 * s, h)), np.zeros((M, h, s)), np.zeros(T * k)
    bx, b1, b2, bg = (np.zeros_like(v) for v in (dx, dW1, dW2, dg))
    mx = np.zeros_like(dx)
    for e, p in experts(idx, M):
        t = p // k
        X, Y, c = x[t], du[t], g[p][:, None]
        ac, n = np.abs(c), len(p)
        G, U, sig, silu, A, eG, eU, e_sig, eA = _hidden(X, W1t[e], s)
        d = Y @ W2t[e]
        ed = (h + 2) * E32 * (np.abs(Y) @ np.abs(W2t[e]))
        ad, aU, aA = np.abs(d), np.abs(U), np.abs(A)
        dg[p] = (A * d).sum(1)
        bg[p] = (eA * ad + aA * ed).sum(1) + (s + 8) * E32 * (aA * ad).sum(1) + TINY
        slope = sig * (1 + G * (1 - sig))
        e_slope = 0.5 * eG + (1 + 2 * np.abs(G)) * e_sig + 8 * E32 * (np.abs(slope) + np.abs(G) * sig)
        dG, dU = c * d * U * slope, c * d * silu
        edG = ac * (ed * aU * np.abs(slope) + ad * eU * np.abs(slope) + ad * aU * e_slope) + 8 * E32 * np.abs(dG)
        edU = ac * (ed * np.abs(silu) + ad * (1.1 * eG + np.abs(G) * e_sig)) + 8 * E32 * np.abs(dU)
        dGU, eGU = np.concatenate([dG, dU], 1), np.concatenate([edG, edU], 1)
        r = eGU + kept * (np.abs(dGU) + eGU)  # with the rounding to bf16
        np.add.at(dx, t, dGU @ W1t[e])
        np.add.at(bx, t, r @ np.abs(W1t[e]))
        np.add.at(mx, t, np.abs(dGU) @ np.abs(W1t[e]))
        dW1[e] = dGU.T @ X
        b1[e] = r.T @ np.abs(X) + (planes * n + 2) * E32 * (np.abs(dGU).T @ np.abs(X))
        gA, egA = c * A, ac * eA + 2 * E32 * ac * aA
        rA = egA + kept * (np.abs(gA) + egA)
        dW2[e] = Y.T @ gA
        b2[e] = np.abs(Y).T @ rA + (planes * n + 2) * E32 * (np.abs(Y).T @ np.abs(gA))
    bx += (2 * planes * s + k + 2) * E32 * mx
    out = [dx, dW1, dW2, dg.reshape(T, k)]
    bounds = [b * (1 + 2 * E16) + E16 * np.abs(v) + TINY for b, v in ((bx, dx), (b1, dW1), (b2, dW2))]
    return out, bounds + [bg.reshape(T, k)]


def _half(resid_bits):
    return E32 if resid_bits == 32 else E16


def block_norm(r, y, w_after, w_before, gate, alpha, eps, norm_after, resid_bits):
    """(r', xn, u) and the bound of each (None where there is none); y [T][k][h] or None."""
    h = r.shape[1]
    u = eu = bu = None
    er = np.zeros_like(r)
    if y is not None:
        u = y.sum(1)
        eu = (y.shape[1] + 1) * E32 * np.abs(y).sum(1)
        bu = eu + E16 * (np.abs(u) + eu) + TINY
        scale = np.ones((len(r), 1)) if gate is None else gate[:, None]
        n, rel = u, 4 * E32
        if norm_after:
            rms = np.sqrt((u * u).mean(1, keepdims=True) + eps)
            n = u / rms
            rel = (h + 16) * E32 + np.sqrt((eu * eu).mean(1, keepdims=True)) / rms
            eu = eu / rms
        w = np.ones(h) if w_after is None else w_after
        b = scale * w * n
        er = np.abs(scale * w) * eu + (rel + 8 * E32) * np.abs(b) + 2 * E32 * np.abs(alpha * r)
        r = alpha * r + b
    br = er + _half(resid_bits) * (np.abs(r) + er) + TINY
    xn = bx = None
    if w_before is not None:
        rms = np.sqrt((r * r).mean(1, keepdims=True) + eps)
        xn = w_before * r / rms
        rel = (h + 16) * E32 + np.sqrt((er * er).mean(1, keepdims=True)) / rms
        bx = np.abs(w_before) * er / rms + rel * np.abs(xn)
        bx = bx + E16 * (np.abs(xn) + bx) + TINY
    return (r, xn, u), (br, bx, bu)


def block_norm_backward(u, r_out, dr_out, dxn, w_after, w_before, gate, alpha, eps, norm_after, resid_bits):
    """(dr, du, dw_after, dw_before, dgate) and the bound of each: every quantity is a short expression of
    sums over a row, so its error is at most (h + 64) E32 times the same expression of magnitudes."""
    T, h = r_out.shape
    c = (h + 64) * E32
    D = np.zeros_like(r_out) if dr_out is None else dr_out.copy()
    mag = np.abs(D)
    dwb = bwb = None
    if dxn is not None:
        rs = 1 / np.sqrt((r_out ** 2).mean(1, keepdims=True) + eps)
        q = dxn * w_before
        D = D + q * rs - r_out * rs ** 3 * (q * r_out).mean(1, keepdims=True)
        mag = mag + np.abs(q) * rs + np.abs(r_out) * rs ** 3 * np.abs(q * r_out).mean(1, keepdims=True)
        dwb = (dxn * r_out * rs).sum(0)
        bwb = (T + h + 64) * E32 * np.abs(dxn * r_out * rs).sum(0) + TINY
    if u is None:
        return ((D, None, None, dwb, None),
                (c * mag + _half(resid_bits) * np.abs(D) + TINY, None, None, bwb, None))
    dr = alpha * D
    br = abs(alpha) * c * mag + _half(resid_bits) * np.abs(dr) * (1 + E16) + TINY
    ru = 1 / np.sqrt((u ** 2).mean(1, keepdims=True) + eps) if norm_after else np.ones((T, 1))
    w = np.ones(h) if w_after is None else w_after
    g = np.ones((T, 1)) if gate is None else gate[:, None]
    p, mp = g * D * w, np.abs(g * w) * mag
    du, md = p * ru, mp * ru
    if norm_after:
        du = du - u * ru ** 3 * (p * u).mean(1, keepdims=True)
        md = md + np.abs(u) * ru ** 3 * (mp * np.abs(u)).mean(1, keepdims=True)
    bu = 3 * c * md + E16 * (np.abs(du) + 3 * c * md) + TINY
    dwa = (g * D * u * ru).sum(0)
    bwa = (T + 2 * h + 128) * E32 * (np.abs(g * u * ru) * mag).sum(0) + TINY
    dgate = bg = None
    if gate is not None:
        dgate = (D * w * u * ru).sum(1)
        bg = 3 * c * (mag * np.abs(w * u * ru)).sum(1) + TINY
    return (dr, du, dwa, dwb, dgate), (br, bu, bwa, bwb, bg)


def clip(grads, max_norm, eps):
    """(norm, scaled gradients)."""
    norm = float(np.sqrt(sum(float((v * v).sum()) for v in grads)))
    c = min(1.0, max_norm / (norm + eps))
    return norm, [v * c for v in grads]
