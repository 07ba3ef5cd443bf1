"""fp64 CPU oracle for the serving operators.

TEST INFRASTRUCTURE ONLY (see :mod:`oracle`). It shares no code with the HIP path.

Conventions: packed rows ``[T, H, D]``, those of sequence b are ``starts[b] .. starts[b + 1] - 1``;
new token i of n stands at position ``lengths[b] - n + i``; position p of sequence b lies in row
``p % page`` of page ``table[b][p // page]`` of a cache ``[pages, Hkv, page, D]``.
"""

from __future__ import annotations

import numpy as np


def rope_ref(x, positions, turns, interleaved=False, amplitude=1.0, transpose=False) -> np.ndarray:
    """Rows x [T, H, D] turned by 2 pi positions turns, the first 2 len(turns) elements of each."""
    x = np.asarray(x, np.float64)
    turns = np.asarray(turns, np.float64)
    rot = 2 * len(turns)
    angle = np.asarray(positions, np.float64)[:, None] * turns
    angle = (angle - np.floor(angle)) * 2 * np.pi
    z = amplitude * np.exp((-1j if transpose else 1j) * angle)[:, None]
    a, b = ((slice(0, rot, 2), slice(1, rot, 2)) if interleaved else
            (slice(0, rot // 2), slice(rot // 2, rot)))
    y = x.copy()
    w = (x[..., a] + 1j * x[..., b]) * z
    y[..., a], y[..., b] = w.real, w.imag
    return y


def token_places(starts, lengths) -> list:
    """(row, sequence, position) of every row that belongs to a sequence."""
    return [(t, b, lengths[b] - starts[b + 1] + t)
            for b in range(len(lengths)) for t in range(starts[b], starts[b + 1])]


def cached_rows(cache, table, b, n) -> np.ndarray:
    """Rows [n, H, D] of positions 0 .. n - 1 of a sequence; NaN where a page does not exist."""
    pages, H, page, D = cache.shape
    out = np.full((n, H, D), np.nan)
    for p in range(n):
        if p // page < table.shape[1] and 0 <= table[b, p // page] < pages:
            out[p] = cache[table[b, p // page], :, p % page]
    return out


def sequence_attention_ref(q, k, v, scale, causal) -> np.ndarray:
    """Rows q [n, Hq, D] over k, v [m, Hkv, D]; with causal, row i sees the keys up to i + m - n."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    n, Hq, D = q.shape
    m, H = k.shape[:2]
    out = np.zeros(q.shape)
    if m == 0:
        return out
    seen = (np.arange(m) <= np.arange(n)[:, None] + m - n) if causal else np.ones((n, m), bool)
    for hq in range(Hq):
        h = hq // (Hq // H)
        x = np.where(seen, q[:, hq] @ k[:, h].T * scale, -np.inf)
        top = x.max(-1, keepdims=True)
        w = np.exp(x - np.where(np.isfinite(top), top, 0.0))
        total = w.sum(-1, keepdims=True)
        out[:, hq] = (w @ v[:, h]) / np.where(total > 0, total, 1.0)
    return out


def packed_attention_ref(q, k, v, starts, k_starts, scale, causal=True) -> np.ndarray:
    out = np.zeros(q.shape)
    for b in range(len(starts) - 1):
        s, e, ks, ke = starts[b], starts[b + 1], k_starts[b], k_starts[b + 1]
        out[s:e] = sequence_attention_ref(q[s:e], k[ks:ke], v[ks:ke], scale, causal)
    return out


def paged_attention_ref(q, k_cache, v_cache, table, lengths, starts, scale) -> np.ndarray:
    """k_cache, v_cache hold the values (codes times scales)."""
    out = np.zeros(q.shape)
    for b, n in enumerate(lengths):
        s, e = starts[b], starts[b + 1]
        out[s:e] = sequence_attention_ref(q[s:e], cached_rows(k_cache, table, b, n),
                                          cached_rows(v_cache, table, b, n), scale, True)
    return out
