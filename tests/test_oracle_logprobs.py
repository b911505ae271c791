"""Pins of the log-probability oracle (oracle/logprobs.py)."""
import numpy as np
import torch

import oracle


def test_against_log_softmax():
    rng = np.random.default_rng(0)
    z = rng.standard_normal((5, 37)) * 3
    z[1, 4:20] = -np.inf
    z[2, [3, 9, 11]] = 7.0
    tokens = np.array([0, 30, 9, -1, 36])
    lp, h, ids, top = oracle.token_logprobs(z, tokens, 0.7, 6)
    ref = torch.log_softmax(torch.from_numpy(z) / 0.7, -1).numpy()
    for r in range(5):
        assert np.isclose(lp[r], 0.0 if tokens[r] < 0 else ref[r, tokens[r]])
        p = np.exp(ref[r])
        assert np.isclose(h[r], -sum(a * b for a, b in zip(p, ref[r]) if a > 0))
        left = list(range(37))
        for j in range(6):
            best = max(left, key=lambda i: (z[r, i], -i))
            assert ids[r, j] == best and np.isclose(top[r, j], ref[r, best])
            left.remove(best)


def test_uniform_and_one_hot():
    z = np.zeros((2, 16))
    z[1, 5] = 1000.0
    lp, h, ids, _ = oracle.token_logprobs(z, np.array([3, 5]), 1.0, 3)
    assert np.allclose(lp, [-np.log(16), 0.0]) and np.allclose(h, [np.log(16), 0.0])
    assert ids.tolist() == [[0, 1, 2], [5, 0, 1]]
