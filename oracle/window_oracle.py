"""CPU oracle for attention with a sliding window and sinks.  TEST INFRASTRUCTURE ONLY.

Key j is visible to query t iff j <= t and (j > t - w or j < sinks): the DMS
mask (arxiv 2506.05345, Fig. 1b) of decisions that are 0 for the first `sinks`
tokens and 1 for the others.  One sequence at a time, dense and in float64.

Beside every result goes `slack`, how far a computation may lie from it whose
products take bf16 operands: probabilities P and score gradients dS rounded to
bf16 (half a step each, 2^-8 of the value), outputs rounded to bf16, the row
term D = dO . out formed from the rounded outputs, and score errors up to
`delta` relative in exp(s) from float32 sums.  With `summed_d` the row term is
sum_j P_j dP_j / sum_j P_j in float32 instead, and no rounding of `out` is allowed
for: weights off by delta, relative, move the mean D of dP by at most 2 delta
sum_j |dS_j|, and the float32 sums of n terms by n half steps of their magnitudes.
"""
from __future__ import annotations

import math

import numpy as np

__all__ = ["window_mask", "window_attention", "window_attention_grads"]

HALF = 2.0 ** -8       # half a bf16 step, relative to the value


def window_mask(T, w, sinks):
    t, j = np.arange(T)[:, None], np.arange(T)[None, :]
    return (j <= t) & ((j > t - w) | (j < sinks))


def _delta(q, k, scale):
    """Relative error of exp(scale q.k) from a float32 sum of d products (each addition half a step
    of at most the sum of magnitudes) and from rounding the exponent."""
    d = q.shape[-1]
    most = scale * float((np.abs(q) @ np.abs(k).T).max()) if q.size and k.size else 0.0
    return (d + 4) * 2.0 ** -24 * most + 2.0 ** -21


def _head(q, k, v, mask, scale):
    s = np.where(mask, scale * (q @ k.T), -np.inf)
    m = s.max(1, keepdims=True)
    e = np.exp(s - m)
    l = e.sum(1, keepdims=True)
    return e / l, (m + np.log(l))[:, 0]


def window_attention(q, k, v, w, sinks, group, scale=None):
    """q [T, Hq, d], k / v [T, Hkv, d] of one sequence: out [T, Hq, d], its slack, lse [Hq, T], its slack."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    T, Hq, d = q.shape
    scale = 1 / math.sqrt(d) if scale is None else scale
    mask = window_mask(T, w, sinks)
    out, slack = np.zeros((T, Hq, d)), np.zeros((T, Hq, d))
    lse, lslack = np.zeros((Hq, T)), np.zeros((Hq, T))
    for hq in range(Hq):
        h = hq // group
        p, lse[hq] = _head(q[:, hq], k[:, h], v[:, h], mask, scale)
        out[:, hq] = p @ v[:, h]
        dl = _delta(q[:, hq], k[:, h], scale)
        slack[:, hq] = (HALF + 3 * dl) * (p @ np.abs(v[:, h])) + HALF * np.abs(out[:, hq])
        lslack[hq] = 2 * dl + 2.0 ** -22 * np.abs(lse[hq])
    return out, slack, lse, lslack


def window_attention_grads(q, k, v, dout, w, sinks, group, scale=None, summed_d=False):
    """Gradients of sum(out * dout): {"dq", "dk", "dv"} and their slacks, one sequence."""
    q, k, v, dout = (np.asarray(x, np.float64) for x in (q, k, v, dout))
    T, Hq, d = q.shape
    scale = 1 / math.sqrt(d) if scale is None else scale
    mask = window_mask(T, w, sinks)
    out, oslack, _, _ = window_attention(q, k, v, w, sinks, group, scale)
    g = {"dq": np.zeros_like(q), "dk": np.zeros_like(k), "dv": np.zeros_like(v)}
    sl = {n: np.zeros_like(x) for n, x in g.items()}
    for hq in range(Hq):
        h = hq // group
        p, _ = _head(q[:, hq], k[:, h], v[:, h], mask, scale)
        do, dl = dout[:, hq], _delta(q[:, hq], k[:, h], scale)
        dp = do @ v[:, h].T
        row = (do * out[:, hq]).sum(1, keepdims=True)
        ds = p * (dp - row)
        near = (d + 4) * 2.0 ** -24 * (np.abs(do) @ np.abs(v[:, h]).T + (np.abs(do) * np.abs(out[:, hq])).sum(1, keepdims=True))
        if summed_d:
            n = mask.sum(1, keepdims=True)
            row_off = 2 * dl * np.abs(ds).sum(1, keepdims=True) + (n + 8) * 2.0 ** -24 * \
                ((p * np.abs(dp)).sum(1, keepdims=True) + np.abs(row)) + (p * near).sum(1, keepdims=True)
        else:
            row_off = (np.abs(do) * oslack[:, hq]).sum(1, keepdims=True)
        ds_off = HALF * np.abs(ds) + 1.01 * p * (row_off + near) + 3 * dl * np.abs(ds)
        g["dv"][:, h] += p.T @ do
        sl["dv"][:, h] += (HALF + 3 * dl) * (p.T @ np.abs(do))
        g["dq"][:, hq] = scale * (ds @ k[:, h])
        sl["dq"][:, hq] = scale * (ds_off @ np.abs(k[:, h]))
        g["dk"][:, h] += scale * (ds.T @ q[:, hq])
        sl["dk"][:, h] += scale * (ds_off.T @ np.abs(q[:, hq]))
    for n in g:
        sl[n] += HALF * (np.abs(g[n]) + sl[n]) + 1e-30
    return g, sl
