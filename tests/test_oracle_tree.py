"""Pins of the drafted-tree oracle (oracle/tree.py)."""
import numpy as np
import pytest

import oracle


def _parents(rng, n):
    return np.array([-1] + [int(rng.integers(-1, i)) for i in range(1, n)])


def test_a_chain_is_the_causal_mask():
    rng = np.random.default_rng(0)
    B, R, Hq, Hkv, D, cap = 2, 4, 4, 2, 8, 16
    q = rng.standard_normal((B, R, Hq, D))
    k, v = rng.standard_normal((2, B, Hkv, cap, D))
    lens = np.array([16, 4])
    want = oracle.verify_attention(q, k, v, lens)
    for b in range(B):
        got = oracle.tree_attention(q[b], k[b, :, :lens[b]], v[b, :, :lens[b]], np.arange(R) - 1)
        assert np.allclose(got, want[b], atol=1e-13)


def test_a_tree_is_one_chain_a_row():
    rng = np.random.default_rng(1)
    n, Hq, Hkv, D, prefix = 9, 4, 1, 8, 5
    parents = _parents(rng, n)
    q, (k, v) = rng.standard_normal((n, Hq, D)), rng.standard_normal((2, Hkv, prefix + n, D))
    got = oracle.tree_attention(q, k, v, parents)
    for i in range(n):
        chain = [i]
        while parents[chain[0]] >= 0:
            chain.insert(0, int(parents[chain[0]]))
        rows = list(range(prefix)) + [prefix + j for j in chain]
        alone = oracle.verify_attention(q[None, [i]], k[None][:, :, rows], v[None][:, :, rows], np.array([len(rows)]))
        assert np.allclose(got[i], alone[0, 0], atol=1e-13)


def test_what_a_row_does_not_see_does_not_reach_it():
    rng = np.random.default_rng(2)
    parents = np.array([-1, 0, 0, 1])
    q, (k, v) = rng.standard_normal((4, 1, 8)), rng.standard_normal((2, 1, 7, 8))
    want = oracle.tree_attention(q, k, v, parents)
    k[0, 3 + 2], v[0, 3 + 2] = np.nan, np.inf
    got = oracle.tree_attention(q, k, v, parents)
    assert np.allclose(got[[0, 1, 3]], want[[0, 1, 3]], atol=1e-13) and np.isnan(got[2]).all()


def test_parents_must_come_earlier():
    for bad in ([-1, 1], [0], [-2], [-1, 0, 3]):
        with pytest.raises(ValueError):
            oracle.tree_sees(bad)


def test_a_chain_accepts_as_the_chain_rule():
    rng = np.random.default_rng(3)
    for _ in range(20):
        z = rng.integers(0, 6, (6, 5)).astype(np.float64)
        tokens = rng.integers(0, 5, 6)
        n_emit, out, star = oracle.accept_greedy(z[None], tokens[None, 1:])
        path, got, best = oracle.accept_tree(z, tokens, np.arange(6) - 1)
        assert path == list(range(int(n_emit[0]))) and got == list(out[0][:n_emit[0]]) and best == list(star[0])


def test_a_tree_accepts_the_longest_agreeing_path():
    z = np.zeros((6, 10))
    for row, best in enumerate([4, 7, 2, 5, 5, 9]):
        z[row, best] = 1.0
    # 0 -> {1: token 3, 2: token 4, 3: token 4}; 2 -> {4: token 2}; 4 -> {5: token 5}
    parents, tokens = [-1, 0, 0, 0, 2, 4], [0, 3, 4, 4, 2, 5]
    assert oracle.accept_tree(z, tokens, parents)[:2] == ([0, 2, 4, 5], [4, 2, 5, 9])
    assert oracle.accept_tree(z, [0, 3, 1, 4, 2, 5], parents)[:2] == ([0, 3], [4, 5])


def test_commit_and_pages():
    rng = np.random.default_rng(4)
    pool = rng.standard_normal((7, 2, 4, 3))
    table = np.array([5, 0, 3])
    rows = oracle.gather_pages(pool, table, 10)
    assert np.array_equal(rows[:, 9], pool[3, :, 1]) and np.array_equal(rows[:, 4], pool[0, :, 0])
    oracle.scatter_rows(pool, table, 6, rng.standard_normal((4, 2, 3)))
    assert np.array_equal(oracle.gather_pages(pool, table, 10)[:, :6], rows[:, :6])
    assert oracle.commit_rows(list("abcdefg"), 4, [0, 2, 3]) == list("abcdfg")
