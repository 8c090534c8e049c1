"""Norm and rotation of queries and keys, fp64 reference (test infrastructure only).

Every head x of D values of a sequence's row i <= gamma_b, at position
t = position_b + i: divided by sqrt(mean(x^2) + eps) and weighted (skipped
without a weight), then every pair (a, c) of the rotated part turned by the
position's angle, (y_a, y_c) -> (y_a cos - y_c sin, y_c cos + y_a sin). The
pairs are (n, n + rot/2), or (2n, 2n + 1) when interleaved.

Status bits as the library's: 1 = gamma_b outside [0, gamma_max]; 128 = a
position outside the table. Rows past gamma_b and the rows of such a sequence
are not outputs (the returned `live` is False there).
"""

from __future__ import annotations

import numpy as np

from .attention import _as_f64

ST_GAMMA = 1
ST_POSITION = 128


def norm_head(x, weight, eps):
    """x [..., D] fp64."""
    if weight is None:
        return x
    return x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * weight


def turn(x, cos, sin, interleaved):
    """x [..., D], cos and sin [rot/2]: the first rot values turned pair by pair."""
    y = np.array(x, copy=True)
    half = len(cos)
    for n in range(half):
        a, c = (2 * n, 2 * n + 1) if interleaved else (n, n + half)
        y[..., a] = x[..., a] * cos[n] - x[..., c] * sin[n]
        y[..., c] = x[..., c] * cos[n] + x[..., a] * sin[n]
    return y


def norm_rope(x, weight, eps, table, position, gamma, interleaved=False):
    """x [B, gmax+1, H, D] (bf16 bits or float), table [max_positions, rot].

    Returns (y fp64, live [B, gmax+1], size fp64, status): size bounds the terms
    that each output is the sum of (|y_a| + |y_c| of its pair before turning).
    """
    x = _as_f64(x)
    w = None if weight is None else _as_f64(weight)
    table = np.asarray(table, dtype=np.float64)
    B, G1, H, D = x.shape
    max_pos, rot = table.shape
    y, size = np.zeros_like(x), np.zeros_like(x)
    live = np.zeros((B, G1), dtype=bool)
    status = 0
    for b in range(B):
        g, p = int(gamma[b]), int(position[b])
        if not 0 <= g < G1:
            status |= ST_GAMMA
            continue
        if not 0 <= p <= max_pos - g - 1:
            status |= ST_POSITION
            continue
        for i in range(g + 1):
            cos, sin = table[p + i, : rot // 2], table[p + i, rot // 2:]
            z = norm_head(x[b, i], w, eps)
            y[b, i] = turn(z, cos, sin, interleaved)
            size[b, i] = np.abs(z)
            for n in range(rot // 2):
                a, c = (2 * n, 2 * n + 1) if interleaved else (n, n + rot // 2)
                size[b, i][:, [a, c]] = (np.abs(z[:, a]) + np.abs(z[:, c]))[:, None]
            live[b, i] = True
    return y, live, size, status
