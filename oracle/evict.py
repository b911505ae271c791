"""Accumulated key weights and eviction (test infrastructure, oracle only).

Parity: pinned (tests/test_oracle_evict.py) by torch's softmax over an explicit mask, by
the weights' total (a row gives 1 to each KV head's query head), and by eviction against
a sort of (weight, index) pairs written the other way round.
"""

import numpy as np


def attention_weights(q, k, lens, committed=None, before=None, decay=1.0, scale=None):
    """decay * before + the softmax weight that keys k [B, Hkv, cap, D] gather from rows
    q [B, R, Hq, D], row i < committed[b] seeing keys 0 .. lens[b] - R + i; the new keys
    bring no weight from before. Returns [B, Hkv, cap], NaN from lens[b] on."""
    B, R, Hq, D = q.shape
    Hkv, cap = k.shape[1], k.shape[2]
    scale = 1.0 / np.sqrt(D) if scale is None else scale
    out = np.full((B, Hkv, cap), np.nan)
    for b in range(B):
        n = int(lens[b])
        for g in range(Hkv):
            w = np.zeros(n)
            if before is not None:
                w[:n - R] = decay * before[b, g, :n - R]
            for i in range(R if committed is None else int(committed[b])):
                for h in range(g * Hq // Hkv, (g + 1) * Hq // Hkv):
                    z = k[b, g, :n - R + i + 1] @ q[b, i, h] * scale
                    e = np.exp(z - z.max())
                    w[:n - R + i + 1] += e / e.sum()
            out[b, g, :n] = w
    return out


def kept_keys(weights, n, keep, sinks, recent):
    """Indices, ascending, of the min(n, keep) of n keys that are kept: the first sinks,
    the last recent, then the largest weights (the lowest index among equals; NaN last)."""
    if n <= keep:
        return np.arange(n)
    fixed = [i for i in range(n) if i < sinks or i >= n - recent]
    rest = [i for i in range(n) if sinks <= i < n - recent]
    rest.sort(key=lambda i: (np.isnan(weights[i]), -weights[i] if not np.isnan(weights[i]) else 0.0, i))
    return np.array(sorted(fixed + rest[:keep - len(fixed)]), dtype=np.int64)
