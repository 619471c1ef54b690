"""Definition of token sampling: integer weights, sorted cuts, a walk by index.  Test infrastructure."""
from __future__ import annotations

import math

import numpy as np

__all__ = ["sample_token"]

UNIT = 2 ** 43


def sample_token(x, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, u=0.0):
    """(token, log-probability) of one row of logits; settings are read as float32."""
    x = np.where(np.isnan(x), -np.inf, np.minimum(np.asarray(x, np.float64), np.finfo(np.float32).max))
    if not (x > -np.inf).any():
        return -1, math.nan
    T, p, least = (float(np.float32(v)) for v in (temperature, top_p, min_p))
    if not T > 0:
        T, top_k = 1.0, 1
    n = len(x)
    k = n if top_k <= 0 else min(top_k, n)
    with np.errstate(invalid="ignore", over="ignore"):
        z = np.where(x == -np.inf, -np.inf, (x - x.max()) / T)
    w = [int(round(v)) for v in np.exp(z) * float(UNIT)]
    order = sorted(range(n), key=lambda i: (-x[i], i))[:k]
    if p < 1:
        want = p * float(sum(w[i] for i in order))
        run, c = 0, 0
        while c < len(order):
            run += w[order[c]]
            c += 1
            if float(run) >= want:
                break
        order = order[:c]
    if least > 0:
        order = [i for i in order if w[i] >= min(least, 1.0) * UNIT]
    total = sum(w[i] for i in order)
    u = 0.0 if not u >= 0 else min(float(np.float32(u)), 1 - 2.0 ** -24)
    run = 0
    for i in sorted(order):
        run += w[i]
        if run > int(u * float(total)):
            return i, float(z[i]) - math.log(total / UNIT)
    raise AssertionError("unreachable")
