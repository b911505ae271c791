"""Pins of the key-weight and eviction oracle (oracle/evict.py)."""
import numpy as np
import torch

import oracle


def test_weights_are_the_masked_softmax():
    rng = np.random.default_rng(0)
    B, R, Hq, Hkv, D, cap = 2, 3, 4, 2, 8, 12
    q, k, before = rng.standard_normal((B, R, Hq, D)), rng.standard_normal((B, Hkv, cap, D)), rng.random((B, Hkv, cap))
    lens = np.array([12, 5])
    got = oracle.attention_weights(q, k, lens, np.array([3, 1]), before, 0.5)
    for b, rows in ((0, 3), (1, 1)):
        n = lens[b]
        z = torch.einsum("rhd,hnd->hrn", torch.from_numpy(q[b]), torch.from_numpy(k[b]).repeat_interleave(2, 0)[:, :n]) / D ** 0.5
        mask = torch.arange(n) > (n - R + torch.arange(R))[:, None]
        p = torch.softmax(z.masked_fill(mask, -torch.inf), -1).view(2, 2, R, n)[:, :, :rows].sum((1, 2)).numpy()
        p[:, :n - R] += 0.5 * before[b, :, :n - R]
        assert np.allclose(got[b, :, :n], p, atol=1e-12) and np.isnan(got[b, :, n:]).all()
    alone = oracle.attention_weights(q, k, lens)
    assert np.allclose(np.nansum(alone, -1), R * Hq / Hkv)


def test_kept_keys_against_pairs():
    rng = np.random.default_rng(1)
    for n, keep, sinks, recent in ((40, 17, 3, 5), (40, 40, 0, 0), (12, 40, 2, 2), (30, 5, 2, 3), (30, 29, 0, 0)):
        w = rng.integers(0, 6, n).astype(np.float64)
        got = oracle.kept_keys(w, n, keep, sinks, recent)
        rank = {i: (2 if i < sinks or i >= n - recent else 1, w[i], -i) for i in range(n)}
        want = sorted(sorted(range(n), key=lambda i: rank[i], reverse=True)[:min(keep, n)])
        assert got.tolist() == want
    assert oracle.kept_keys(np.array([np.nan, -np.inf, 0.0]), 3, 2, 0, 0).tolist() == [1, 2]
