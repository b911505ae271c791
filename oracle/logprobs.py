"""Log probabilities of given tokens, entropy and top alternatives (test
infrastructure, oracle only).

Parity: pinned (tests/test_oracle_logprobs.py) by torch's log_softmax in float64, by the
entropies of uniform and one-hot rows, and by a brute-force order of the alternatives.
"""

import numpy as np


def token_logprobs(z, tokens, temperature=1.0, top_n=0):
    """z [N, V], tokens [N] (-1: none). Returns (logprob [N], entropy [N], ids [N, top_n],
    logprobs [N, top_n]): equal logits by the lowest index; a token -1 gives 0."""
    z = np.asarray(z, dtype=np.float64) + 0.0
    N, V = z.shape
    logprob, entropy = np.zeros(N), np.empty(N)
    ids, lps = np.empty((N, top_n), dtype=np.int64), np.empty((N, top_n))
    for r in range(N):
        x = (z[r] - z[r].max()) / temperature
        lse = np.log(np.exp(x).sum())
        lp = x - lse
        p = np.exp(lp)
        entropy[r] = -(p[p > 0] * lp[p > 0]).sum()
        if tokens[r] >= 0:
            logprob[r] = lp[tokens[r]]
        ids[r] = sorted(range(V), key=lambda i: (-z[r, i], i))[:top_n] if V <= 4096 else np.lexsort((np.arange(V), -z[r]))[:top_n]
        lps[r] = lp[ids[r]]
    return logprob, entropy, ids, lps
