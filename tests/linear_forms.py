"""The forms in which the linear maps and their gradients run, from the plan that the library reports, and for each two shapes of
a fixed set, one of least work and one of many times it (no GPU needed: plans are host queries).

A form is what the kernels are instantiated for:
  ("linear" or "q8", rows of a tile, columns, stages, listed)       rows 0: without tiles, columns of a workgroup
  ("dx", rows, columns, listed, one entry per token)                dx alone, and beside dW where they do not share a launch
  ("dW", rows, columns, in runs, along the rows)                    the same of dW
  ("both", rows of dx's tile, rows and columns of dW's, in runs, one entry per token)   both in one launch
"""
from __future__ import annotations

import functools

import numpy as np


def forms(kind, T, K, N, M, k):
    from paper_2609_36301_amd import expert_linear_plan
    p = expert_linear_plan(T, K, N, M, k, kind)
    if kind != "backward":
        return [(kind, p["tile_rows"], p["cols"], p["stages"], bool(p["listed"]))]
    rows, cols, runs = p["dw_rows"], p["dw_cols"], p["dw_runs"] > 1
    along = cols == 64 or (rows == cols == 128 and bool(p["listed"]) and K <= 128 and N > 128)
    found = [("dx", p["tile_rows"], p["cols"], bool(p["listed"]), k == 1), ("dW", rows, cols, runs, along)]
    if not p["listed"] and cols < 256:
        found.append(("both", p["tile_rows"], rows, cols, runs, k == 1))
    return found


def expected():
    two = (False, True)
    out = []
    for kind in ("linear", "q8"):
        out += [(kind, 0, 16, 0, False), (kind, 0, 256, 0, False), (kind, 256, 256, 2, True), (kind, 32, 128, 2, True)]
        for rows, stages in ((32, 3), (64, 3), (128, 2)):
            out += [(kind, rows, cols, stages, listed) for cols in (64, 128) for listed in two]
    out += [("dx", rows, cols, listed, one) for rows in (32, 64, 128) for cols in (64, 128) for listed in two for one in two]
    out += [("dx", 256, 256, True, one) for one in two]
    out += [("dW", 128, 64, runs, True) for runs in two] + [("dW", 64, 128, runs, False) for runs in two]
    out += [("dW", 128, 128, runs, along) for runs in two for along in two] + [("dW", 256, 256, False, False)]
    out += [("both", bm, r, c, runs, one) for bm in (32, 64, 128) for r, c in ((128, 64), (64, 128), (128, 128)) for runs in two
            for one in two]
    return out


@functools.lru_cache(None)
def shapes():
    """{form: [(T, K, N, M, k) of least work, of most work up to 1.5e9]} over 60000 shapes per kind."""
    rng = np.random.default_rng(1)

    def draw(lo, hi, step=1):
        return step * int(round(np.exp(rng.uniform(np.log(lo / step), np.log(hi / step)))))

    least, most = {}, {}
    for kind, step in (("linear", 8), ("backward", 8), ("q8", 16)):
        for _ in range(60000):
            n, M, k = draw(1, 300000), draw(1, 2000), int(rng.choice([1, 1, 2, 3, 8]))
            K, N = draw(step, 2048, step), draw(8, 2048, 8)
            T = max(1, n // k)
            work = (T * k + 40 * M) * K * N + 2000 * T * k
            if work > 4e9 or M * K * N > 1 << 27 or T * k * (K + N) > 1 << 28:
                continue
            for form in forms(kind, T, K, N, M, k):
                if form not in least or work < least[form][0]:
                    least[form] = work, (T, K, N, M, k)
                if work < 1.5e9 and (form not in most or work > most[form][0]):
                    most[form] = work, (T, K, N, M, k)
    return {form: [shape] + ([most[form][1]] if form in most else []) for form, (_, shape) in least.items()}


def ids(form):
    return "-".join(str(int(f)) if not isinstance(f, str) else f for f in form)
