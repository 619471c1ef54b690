"""CPU oracle for rotary positions with several axes.  TEST INFRASTRUCTURE ONLY.

Pair i of a token turns by pos[axis(i)] * inv_freq[i] as a complex number; all in
float64.  With `borrow`, element 0 of the first query head of each group is taken
as the decision neuron (arxiv 2506.05345, App. C) and zeroed before the rotation.
"""
from __future__ import annotations

import numpy as np

__all__ = ["rope_axes", "rope_rotate", "rope_borrow"]


def rope_axes(sections, interleaved):
    """Axis of every pair."""
    if not interleaved:
        return [a for a, n in enumerate(sections) for _ in range(n)]
    A = len(sections)
    return [i % A if i // A < sections[i % A] else 0 for i in range(sum(sections))]


def rope_rotate(x, positions, inv_freq, axes, rotary_dim, offset=0, adjacent=False, factor=1.0, back=False):
    """x [T, heads, d], positions [A, T] -> rotated copy (the transposed rotation with `back`)."""
    y = np.array(x, np.float64)
    half = rotary_dim // 2
    i = np.arange(half)
    lo = offset + (2 * i if adjacent else i)
    hi = lo + (1 if adjacent else half)
    angle = np.asarray(positions, np.float64)[axes].T * np.asarray(inv_freq, np.float64)
    z = (y[..., lo] + 1j * y[..., hi]) * factor * np.exp((-1j if back else 1j) * angle)[:, None]
    y[..., lo], y[..., hi] = z.real, z.imag
    return y


def rope_borrow(q, group):
    """(logits [T, Hkv], q with the borrowed neurons zeroed)."""
    q = np.array(q, np.float64)
    logits = q[:, ::group, 0].copy()
    q[:, ::group, 0] = 0
    return logits, q
