"""The distillation loss where a teacher's entries cover most classes (V <= 2 k), to 60 digits, and how far a result may be
from it.

There P and Q come close as the temperature grows, and tau^2 KL is made of what is left of their difference.  The kernel
writes e^x as n + r, n whole, with n = 1 and r = e^x - 1 for |x| <= 1/2, else n = 0 and r = e^x; sums the whole parts exactly; and takes
   D_e = Z U (P_e - Q_e) = (n_e Nu - n'_e Nz) + n_e B - n'_e A + r_e U - r'_e Z,   Z = Nz + A, U = Nu + B
(n', r' of the class's entries together).  The bounds follow that, with E = 2^-24:
   r       (12 + 3 |x|) E |r|             (difference, factor, product; eight terms of a series, or an exponential)
   sums    80 E of the sum of magnitudes  (chains of up to 64 terms, and the joining of 256 threads)
   others  E of the result each
"""
from __future__ import annotations

import decimal
import math
from decimal import Decimal

import numpy as np

from layer_ref import E16, E32, TINY

D0 = Decimal(0)
INF = float("inf")


def _exp(x):
    return D0 if x == Decimal("-Infinity") else x.exp()


def _parts(d, tau):
    """(whole part, rest, e^x, bound of the rest) of x = d / tau."""
    if d == -INF:
        return 0, 0.0, D0, 0.0
    x = Decimal(d) / Decimal(tau)
    e = _exp(x)
    whole = int(abs(x) <= Decimal("0.5"))
    rest = float(e - whole)
    return whole, rest, e, (12 + 3 * abs(float(x))) * E32 * abs(rest)


def distill(z, ids, values, tau, weight=None, bits=32):
    """loss [T], gradient [T][V], and their bounds."""
    T, V = z.shape
    half = E32 if bits == 32 else E16
    loss, grad = np.zeros(T), np.zeros((T, V))
    bl, bg = np.full(T, TINY), np.full((T, V), TINY)
    with decimal.localcontext() as ctx:
        ctx.prec = 60
        ctx.Emin, ctx.Emax = decimal.MIN_EMIN, decimal.MAX_EMAX
        for t in range(T):
            w = 1.0 if weight is None else float(weight[t])
            valid = [j for j in range(ids.shape[1]) if 0 <= ids[t, j] < V and values[t, j] != -INF]
            if not valid:
                continue
            m, top = z[t].max(), max(values[t, j] for j in valid)
            n, r, e, er = (list(v) for v in zip(*[_parts(float(v - m), tau) for v in z[t]]))
            n2, r2, e2, er2 = (list(v) for v in zip(*[_parts(float(values[t, j]) - float(top), tau) for j in valid]))
            Z, U, Nz, Nu = sum(e), sum(e2), sum(n), sum(n2)
            A, B, fZ, fU = float(Z - Nz), float(U - Nu), float(Z), float(U)
            eA = sum(er) + 80 * E32 * sum(map(abs, r))
            eB = sum(er2) + 80 * E32 * sum(map(abs, r2))
            eZ, eU = eA + E32 * fZ, eB + E32 * fU

            def difference(c, whole, rest, erest):
                """bound of D of class c against entries of these whole parts, rests and bounds of the rests"""
                kept = abs(n[c] * Nu - whole * Nz) + n[c] * abs(B) + whole * abs(A) + abs(r[c]) * fU + abs(rest) * fZ
                return n[c] * eB + whole * eA + er[c] * fU + abs(r[c]) * eU + erest * fZ + abs(rest) * eZ + 8 * E32 * kept

            total, bound, left, count = D0, 0.0, D0, [0] * V
            size = Decimal(tau) ** 2
            for i, j in enumerate(valid):
                c = int(ids[t, j])
                count[c] += 1
                q, p = e2[i] / U, e[c] / Z
                fq, fp = float(q), float(p)
                if q == 0:
                    total += p
                elif p == 0:
                    total += Decimal("Infinity")
                else:
                    total += q * (q / p).ln() - q + p
                gone = (eU / fU + (16 + er2[i] / E32 / max(abs(r2[i]), 1e-300)) * E32)  # relative error of q
                away = (eZ / fZ + (16 + er[c] / E32 / max(abs(r[c]), 1e-300)) * E32)    # and of p
                if n[c] and n2[i]:
                    ratio = float(q / p)
                    delta = float(q / p - 1)
                    ed = difference(c, 1, r2[i], er2[i]) / (fU * float(e[c])) + abs(delta) * (away + gone)
                    log = abs(math.log(ratio))
                    phi = float(q / p * (q / p).ln() - q / p + 1)
                    bound += fp * (log + ed) * ed + fp * abs(phi) * (away + 32 * E32)
                    if abs(delta) > 0.1:  # (by its logarithm)
                        bound += fp * E32 * (16 * ratio * log + 16 * abs(delta) + 4 * ratio)
                elif p > 0:
                    ln = abs(math.log(fZ)) + abs(math.log(fU))
                    far = (abs(float(values[t, j]) - float(top)) + abs(float(z[t, c] - m))) / tau
                    bound += fq * (eZ / fZ + eU / fU + 8 * E32 * (ln + far + 1) + (ln + far) * gone) + fp * away + fq * gone
            left = sum((1 - count[c]) * e[c] for c in range(V)) / Z
            rest = sum(abs(1 - count[c]) * (er[c] + 80 * E32 * abs(r[c])) for c in range(V)) / fZ
            total = size * (total + left)
            loss[t] = float(total)
            bound += rest + abs(float(left)) * (eZ / fZ + 8 * E32)
            whole = sum(abs(1 - count[c]) * float(e[c]) for c in range(V)) / fZ
            bound += 80 * E32 * (abs(float(total / size)) + 2 * whole)
            bl[t] += float(size) * bound if math.isfinite(bound) else 0.0
            # the gradient
            for c in range(V):
                mine = [i for i, j in enumerate(valid) if ids[t, j] == c] if count[c] else []
                Q = sum((e2[i] for i in mine), D0) / U
                g = float(Decimal(w) * Decimal(tau) * (e[c] / Z - Q))
                grad[t, c] = g
                if mine:
                    erest = sum(er2[i] for i in mine) + 80 * E32 * sum(abs(r2[i]) for i in mine)
                    ed = difference(c, sum(n2[i] for i in mine), sum(r2[i] for i in mine), erest)
                    b = abs(w) * tau * ed / (fZ * fU) + abs(g) * (eZ / fZ + eU / fU + 8 * E32)
                else:
                    b = abs(g) * (eZ / fZ + (16 + er[c] / E32 / max(abs(r[c]), 1e-300)) * E32)
                bg[t, c] += b * (1 + E16) + half * abs(g)
    return (loss, grad), (bl, bg)
