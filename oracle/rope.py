"""fp64 rotary positions.  TEST INFRASTRUCTURE ONLY (see the package docstring)."""
from __future__ import annotations

import numpy as np


def grid_positions(n, grid, origin=(0, 0, 0)):
    """Positions [3, n] of a row-major (T, H, W) grid's tokens, and which of the n
    tokens lie in it."""
    t, h, w = grid
    idx = np.arange(n)
    pos = np.stack([idx // (h * w) + origin[0], idx // w % h + origin[1], idx % w + origin[2]])
    return pos, idx < t * h * w


def rotate(x, positions, freq, pairs, interleaved, inverse=False, turned=None):
    """x [N, H, d] float64 with positions [axes, N]; tokens with turned False stay."""
    P = sum(pairs)
    out = x.copy()
    axis = np.repeat(np.arange(len(pairs)), pairs)
    for n in range(x.shape[0]):
        if turned is not None and not turned[n]:
            continue
        for i in range(P):
            t = float(positions[axis[i]][n]) * float(freq[i]) * (-1.0 if inverse else 1.0)
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + P)
            c, s = np.cos(t), np.sin(t)
            out[n, :, a] = x[n, :, a] * c - x[n, :, b] * s
            out[n, :, b] = x[n, :, a] * s + x[n, :, b] * c
    return out
