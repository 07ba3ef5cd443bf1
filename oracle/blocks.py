"""fp64 CPU oracle for the long-context operators.

TEST INFRASTRUCTURE ONLY (see :mod:`oracle`). It shares no code with the HIP path.

Conventions: sequence b has ``lengths[b]`` valid keys (all of them without lengths), query i of
it sits at key ``n_i = i + len_b - Sq``, block n of ``block`` keys holds keys
``[n * block, (n + 1) * block)``.
"""

from __future__ import annotations

import numpy as np


def _lengths(lengths, B, Skv):
    if lengths is None:
        return [Skv] * B
    return [min(max(int(n), 0), Skv) for n in lengths]


def block_summary_ref(k, block, lengths=None) -> np.ndarray:
    """Mean of each block's valid keys [B, Hkv, NB, D]; 0 for a block without one."""
    k = np.asarray(k, np.float64)
    B, H, S, D = k.shape
    nb = -(-S // block)
    out = np.zeros((B, H, nb, D))
    for b, n in enumerate(_lengths(lengths, B, S)):
        for j in range(0, n, block):
            out[b, :, j // block] = k[b, :, j:min(j + block, n)].mean(1)
    return out


def block_select_ref(q, summary, Skv, topk, block, sinks, local, lengths=None) -> np.ndarray:
    """Blocks of each query [B, Hkv, Sq, topk], ascending, filled with -1."""
    q, m = np.asarray(q, np.float64), np.asarray(summary, np.float64)
    B, Hq, Sq, D = q.shape
    H = m.shape[1]
    G = Hq // H
    out = np.full((B, H, Sq, topk), -1, np.int64)
    for b, n in enumerate(_lengths(lengths, B, Skv)):
        for h in range(H):
            for i in range(Sq):
                d = i + n - Sq
                if d < 0:
                    continue
                cur = d // block
                if cur + 1 <= topk:
                    out[b, h, i, :cur + 1] = np.arange(cur + 1)
                    continue
                with np.errstate(invalid="ignore"):
                    x = q[b, h * G:(h + 1) * G, i] @ m[b, h, :cur + 1].T
                x = np.where(np.isnan(x), -np.inf, x).max(0)
                forced = [j for j in range(cur + 1) if j < sinks or j > cur - local]
                rest = [j for j in range(cur + 1) if j not in set(forced)]
                rest.sort(key=lambda j: (-x[j], j))
                out[b, h, i] = sorted(forced + rest[:topk - len(forced)])
    return out


def _softmax_rows(q, k, v, seen, scale):
    x = (q @ k.T) * scale
    x = np.where(seen, x, -np.inf)
    top = x.max(-1, keepdims=True, initial=-np.inf)
    w = np.exp(x - np.where(np.isfinite(top), top, 0.0))
    total = w.sum(-1, keepdims=True)
    return (w @ v) / np.where(total > 0, total, 1.0)


def attention_blocks_ref(q, k, v, blocks, block, scale, lengths=None) -> np.ndarray:
    """Attention [B, Hq, Sq, D] of each query over the keys up to its own that lie in a block of
    its list (of its sequence and kv head)."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    blocks = np.asarray(blocks)
    B, Hq, Sq, D = q.shape
    H, S = k.shape[1], k.shape[2]
    G = Hq // H
    out = np.zeros(q.shape)
    for b, n in enumerate(_lengths(lengths, B, S)):
        key = np.arange(n)
        for h in range(H):
            for i in range(Sq):
                seen = np.isin(key // block, blocks[b, h, i]) & (key <= i + n - Sq)
                if not seen.any():
                    continue
                rows = slice(h * G, (h + 1) * G)
                out[b, rows, i] = _softmax_rows(q[b, rows, i], k[b, h, :n][seen],
                                                v[b, h, :n][seen], True, scale)
    return out


def shared_prefix_ref(q, kp, vp, k, v, scale, causal=True, lengths=None) -> np.ndarray:
    """Attention [B, Hq, Sq, D] of each sequence over the keys of the prefix, then its own."""
    q, kp, vp, k, v = (np.asarray(t, np.float64) for t in (q, kp, vp, k, v))
    B, Hq, Sq, D = q.shape
    H, S, Lp = k.shape[1], k.shape[2], kp.shape[1]
    G = Hq // H
    out = np.zeros(q.shape)
    for b, n in enumerate(_lengths(lengths, B, S)):
        diag = np.arange(Sq) + Lp + n - Sq
        seen = np.arange(Lp + n) <= diag[:, None] if causal else np.ones((Sq, Lp + n), bool)
        for hq in range(Hq):
            h = hq // G
            out[b, hq] = _softmax_rows(q[b, hq], np.concatenate([kp[h], k[b, h, :n]]),
                                       np.concatenate([vp[h], v[b, h, :n]]), seen, scale)
    return out
