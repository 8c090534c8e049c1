"""Verification attention with a sliding window and sinks, fp64 reference
(test infrastructure only).

As attention.verify_attention, but the row at cache position pos sees, of the
keys j <= pos with mask 1, those with j > pos - window or j < sinks (window 0:
all of them).
"""

from __future__ import annotations

import numpy as np

from .attention import _as_f64, attend_rows, sequence_status


def visible(kv_len_b, gamma_b, window, sinks, mask_b=None):
    """bool [gamma_b + 1, kv_len_b]."""
    j = np.arange(kv_len_b)
    pos = kv_len_b - (gamma_b + 1) + np.arange(gamma_b + 1)
    see = j[None, :] <= pos[:, None]
    if window > 0:
        see = see & ((j[None, :] > pos[:, None] - window) | (j[None, :] < sinks))
    if mask_b is not None:
        see = see & (np.asarray(mask_b[:kv_len_b]) != 0)[None, :]
    return see


def verify_attention(q, k_cache, v_cache, kv_len, gamma, scale, mask=None, window=0, sinks=0):
    """Arguments as attention.verify_attention (bf16 bits or floats). Returns
    (out [B, gmax+1, Hq, D], size of the same shape, status): size is the same
    average of |v|, which bounds what a relative error of the weights can do."""
    q = np.asarray(q)
    B, G1, Hq, D = q.shape
    Hkv, cap = k_cache.shape[1], k_cache.shape[2]
    grp = Hq // Hkv
    out, size = np.zeros((B, G1, Hq, D)), np.zeros((B, G1, Hq, D))
    status = 0
    for b in range(B):
        st = sequence_status(int(kv_len[b]), int(gamma[b]), G1 - 1, cap)
        status |= st
        if st:
            continue
        L, n = int(kv_len[b]), int(gamma[b]) + 1
        see = visible(L, n - 1, window, sinks, None if mask is None else mask[b])
        used = np.flatnonzero(see.any(0))  # entries that no row sees are never read
        rows = np.repeat(see[:, used], grp, axis=0)
        for g in range(Hkv):
            K, V = _as_f64(k_cache[b, g, used]), _as_f64(v_cache[b, g, used])
            heads = slice(g * grp, (g + 1) * grp)
            Q = _as_f64(q[b, :n, heads]).reshape(n * grp, D)
            out[b, :n, heads] = attend_rows(Q, K, V, rows, scale).reshape(n, grp, D)
            size[b, :n, heads] = attend_rows(Q, K, np.abs(V), rows, scale).reshape(n, grp, D)
    return out, size, status
