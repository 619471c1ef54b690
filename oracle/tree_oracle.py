"""Float64 definitions of the calls on trees of drafted tokens.  Test infrastructure."""
from __future__ import annotations

import numpy as np

__all__ = ["tree_paths", "tree_attention", "tree_accept"]


def tree_paths(parents):
    """For every node the list of nodes from its root to itself."""
    paths = []
    for x, p in enumerate(parents):
        assert -1 <= p < x
        paths.append((paths[p] if p >= 0 else []) + [x])
    return paths


def tree_attention(q, k, v, flags, parents, pos, w, group, cache_k, cache_v, cache_pos, cache_flag, scale=None):
    """One sequence.  q [m, Hq, d], k, v [m, Hkv, d], flags [m, Hkv]: the nodes' rows; cache_*[h]: the retained keys,
    values, positions and flags of KV head h.  Returns (out, slack): the outputs, and for every element how far a
    bf16 result may be from it whose weights were rounded to bf16:
      weights p (1 + a), |a| <= 2^-8, divided by their own sum, move the output by at most
      2^-8 / (1 - 2^-8) sum p |v - out|;
      a score in float32 (d products and sums of bf16 operands) is off by at most (d + 8) 2^-24 sum |q k| scale, its
      exponential by 2^-20 more, and the weights by twice that;
      sums over the keys add 2^-24 a step, 2^-14 for fewer than 1024 tiles of float32 sums, of sum p |v|;
      the output is rounded once, 2^-8 of it."""
    m, Hq, d = q.shape
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    paths = tree_paths(parents)
    out, slack = np.zeros((m, Hq, d)), np.zeros((m, Hq, d))
    for x, path in enumerate(paths):
        t = pos + len(path) - 1
        for h in range(k.shape[1]):
            seen = [j for j in range(len(cache_pos[h])) if not cache_flag[h][j] or cache_pos[h][j] > t - w]
            mine = [a for z, a in enumerate(path) if not flags[a, h] or pos + z > t - w]
            kk = np.concatenate([cache_k[h][seen], k[mine, h]])
            vv = np.concatenate([cache_v[h][seen], v[mine, h]])
            for qh in range(h * group, (h + 1) * group):
                s = kk @ q[x, qh] * scale
                p = np.exp(s - s.max())
                p /= p.sum()
                o = p @ vv
                off = (d + 8) * 2.0 ** -24 * scale * (np.abs(kk) @ np.abs(q[x, qh])).max() + 2.0 ** -20
                spread = p @ np.abs(vv - o)
                lim = (2.0 ** -8 / (1 - 2.0 ** -8) + 2 * off) * spread + 2.0 ** -14 * (p @ np.abs(vv))
                out[x, qh] = o
                slack[x, qh] = lim + 2.0 ** -8 * (np.abs(o) + lim) + 1e-30
    return out, slack


def tree_accept(parents, tokens, targets, first=None):
    """(path, next token) of one tree."""
    path, at, want = [], -1, first
    while True:
        kids = [x for x in range(at + 1, len(parents)) if parents[x] == at and (want is None or tokens[x] == want)]
        if not kids:
            return path, -1 if want is None else int(want)
        at = kids[0]
        path.append(at)
        want = targets[at]
