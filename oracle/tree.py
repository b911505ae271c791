"""Drafted trees over a paged cache: append, attention, greedy acceptance and commit,
float64 (test infrastructure, oracle only).

A tree has n rows: row 0 is the last committed token, parents[i] < i the row that row i
follows, -1 the prefix. Row i sees the prefix, its ancestors and itself; a chain
(parents[i] = i - 1) is the causal mask of verify_attention. A paged cache keeps row m of
scene b as row m % page of page table[b][m // page].

Parity: pinned (tests/test_oracle_tree.py): chains against verify_attention and
accept_greedy, trees against one chain a leaf, commits against a list of rows.
"""

import numpy as np


def gather_pages(pool, table_row, n):
    """Rows 0 .. n - 1 of one scene from a pool [pages, Hkv, page, D]: [Hkv, n, D]."""
    page = pool.shape[2]
    rows = pool[table_row[:-(-n // page)]]                     # [pages, Hkv, page, D]
    return np.swapaxes(rows, 0, 1).reshape(pool.shape[1], -1, pool.shape[3])[:, :n]


def scatter_rows(pool, table_row, first, rows):
    """Write rows [n, Hkv, D] at first .. first + n - 1 of one scene, in place."""
    page = pool.shape[2]
    for i in range(len(rows)):
        at = first + i
        pool[table_row[at // page], :, at % page] = rows[i]


def tree_sees(parents):
    """[n, n] truth values: row j is row i or an ancestor of it."""
    n = len(parents)
    sees = np.zeros((n, n), dtype=bool)
    for i, p in enumerate(parents):
        if not -1 <= p < i:
            raise ValueError("a parent must be an earlier row or -1")
        if p >= 0:
            sees[i] = sees[p]
        sees[i, i] = True
    return sees


def tree_attention(q, k, v, parents, scale=None, spread=False):
    """One scene: q [n, Hq, D], k and v [Hkv, prefix + n, D], parents [n] -> [n, Hq, D].

    What a row does not see has no part in its sums. spread: also a bound on
    sum_j w_j |v_j - o| (what an error of one part in the weights can move the output by),
    the root of sum_j w_j (v_j - o)^2, and the largest sum of |q k| scale (what an error
    of one part in a product can move a score by)."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    n, hq, d = q.shape
    hkv, keys, _ = k.shape
    if scale is None:
        scale = 1.0 / np.sqrt(d)
    prefix = keys - n
    visible = np.concatenate([np.ones((n, prefix), dtype=bool), tree_sees(parents)], axis=1)
    out, dev, size = np.zeros_like(q), np.zeros_like(q), np.zeros((n, hq, 1))

    def rows(i, h, kk, vv, seen):  # rows i of head h over keys of which they see some
        s = np.where(seen, (q[i, h] @ kk.T) * scale, -np.inf)
        w = np.exp(s - s.max(axis=1, keepdims=True))
        w = w / w.sum(axis=1, keepdims=True)
        o = w @ vv
        out[i, h] = o
        if spread:
            dev[i, h] = np.sqrt(np.maximum(w @ (vv * vv) - o * o, 0.0))
            size[i, h] = np.where(seen, np.abs(q[i, h]) @ np.abs(kk).T, 0.0).max(axis=1, keepdims=True) * scale

    with np.errstate(invalid="ignore", over="ignore"):
        for h in range(hq):
            g = h // (hq // hkv)
            if np.isfinite(k[g]).all() and np.isfinite(v[g]).all():
                rows(np.arange(n), h, k[g], v[g], visible)
                continue
            for i in range(n):
                rows(np.array([i]), h, k[g][visible[i]], v[g][visible[i]], np.ones((1, int(visible[i].sum())), dtype=bool))
    return (out, dev, size) if spread else out


def accept_tree(logits, tokens, parents):
    """One scene: logits [n, V], tokens [n], parents [n] -> (path, out, argmax)."""
    n = len(tokens)
    star = [int(np.flatnonzero(np.asarray(z) == np.max(z))[0]) for z in logits]
    path, out = [], []
    at = 0 if n else None
    while at is not None:
        path.append(at)
        out.append(star[at])
        at = next((c for c in range(at + 1, n) if parents[c] == at and tokens[c] == star[at]), None)
    return path, out, star


def commit_rows(rows, n_new, path):
    """A scene's rows (a list) after a commit: the prefix, then the path's."""
    first = len(rows) - n_new
    return rows[:first] + [rows[first + p] for p in path]
