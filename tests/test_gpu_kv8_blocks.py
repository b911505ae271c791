"""Every block of 32 keys counts once in the attention over the 8-bit cache, at every
cluster size and in even shares: each row has one key that holds three quarters of its weight, in a
block of its own, with a value of its own. A block lost or taken twice is an error of
several times the tolerance (checked on the reference)."""
import numpy as np
import pytest
import torch

import oracle
from paper_2606_31160_gb300 import sd, workloads
from tests.helpers import ensure_lib, to64

pytestmark = pytest.mark.gpu

SCALE = 2.0 ** -7


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_lib()
    sd.get_device_error()
    yield
    sd.set_cluster_size(0)


def _softmax(z):
    e = np.exp(z - z.max())
    return e / e.sum()


def _planted(n, D, seed):
    """Codes of keys and values [n, D], query rows [blocks, D]; row r's key lies in block r
    of 32 keys (the last one short)."""
    rng = np.random.default_rng(seed)
    blocks = -(-n // 32)
    assert blocks <= min(D, 128)
    k = oracle.round_e4m3(rng.standard_normal((n, D)) * 20)
    v = oracle.round_e4m3(np.clip(rng.standard_normal((n, D)) * 100, -448, 448))
    q = rng.standard_normal((blocks, D)) * 0.3
    q = workloads.to_bf16(q.astype(np.float32)).float().numpy().astype(np.float64)
    at = np.array([min(32 * r + int(rng.integers(0, 32)), n - 1) for r in range(blocks)])
    k[at] = 0.0
    k[at, np.arange(blocks)] = 448.0
    v[at] = 448.0 * rng.choice([-1.0, 1.0], (blocks, D))
    for r in range(blocks):
        z = k @ q[r] * SCALE / np.sqrt(D)
        rest = np.exp(z).sum() - np.exp(z[at[r]])
        q[r, r] = np.log(3 * rest) * np.sqrt(D) / (448 * SCALE)
    return k, v, workloads.to_bf16(q.astype(np.float32))


def _reference(k, v, q):
    """(rows, their tolerances); a block that is lost or counts twice is seen."""
    k, v, q = k * SCALE, v * SCALE, to64(q)
    n, D = k.shape
    ref, tol = np.empty(q.shape), np.empty(q.shape)
    for r in range(len(q)):
        p = _softmax(k @ q[r] / np.sqrt(D))
        ref[r] = p @ v
        # the output's rounding (2^-9 of it, doubled) and six standard deviations of the
        # weights' (8 significant bits; a small one's 2^-21 of the row's sum)
        tol[r] = 2.0 ** -8 * np.abs(ref[r]) + 6 * 2.0 ** -9 / np.sqrt(3) * np.sqrt(p ** 2 @ v ** 2) + \
            6 * 2.0 ** -21 * np.sqrt((v ** 2).sum(0))
        for count in (0.0, 2.0):
            w = p.copy()
            w[32 * r:32 * r + 32] *= count
            assert np.any(np.abs(w @ v / w.sum() - ref[r]) > 3 * tol[r])
    return ref, tol


@pytest.mark.parametrize("cs", [0, 1, 2, 4, 6, 8, 16])
@pytest.mark.parametrize("n,D", [(3001, 128), (4096, 128), (2037, 64), (1025, 64)])
def test_every_block_at_every_cluster_size(n, D, cs):
    k, v, q = _planted(n, D, n)
    ref, tol = _reference(k, v, q)
    c = sd.KV8Cache.empty(1, 1, n, D, 32)
    for t, x in ((c.k, k), (c.v, v)):
        t.copy_(torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).cuda().view(1, 1, n, D))
    c.k_scale.fill_(SCALE)
    c.v_scale.fill_(SCALE)
    c.len.fill_(n)
    sd.set_cluster_size(cs)
    try:
        out = to64(sd.kv8_attention(q.cuda().view(1, 1, -1, D), c))[0, 0]
    finally:
        sd.set_cluster_size(0)
    assert np.all(np.abs(out - ref) <= tol), (np.abs(out - ref) - tol).max(axis=1)
    assert sd.get_device_error() == 0


@pytest.mark.parametrize("n,D", [(3001, 128), (2037, 64)])
def test_every_block_in_even_shares(n, D):
    """Scenes of one to all of the blocks; a scene's own blocks among its rows are checked."""
    k, v, q = _planted(n, D, n + 1)
    blocks = len(q)
    B = next(b for b in range(16, 200) if sd.kv8_attention_workspace_bytes(b, 1, blocks, 1, D, n) > 0)
    rng = np.random.default_rng(n)
    lens = rng.integers(n // 2, n + 1, B)
    lens[0], lens[1] = n, 1 + n // 2
    c = sd.KV8Cache.empty(B, 1, n, D, 32)
    for t, x in ((c.k, k), (c.v, v)):
        x = torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).cuda().view(torch.uint8)
        t.copy_(x.expand(B, 1, n, D).contiguous().view(torch.float8_e4m3fn))
    c.k_scale.fill_(SCALE)
    c.v_scale.fill_(SCALE)
    c.len.copy_(torch.from_numpy(lens.astype(np.int32)))
    out = to64(sd.kv8_attention(q.cuda().expand(B, 1, blocks, D).contiguous(), c))[:, 0]
    for b in range(B):
        at = 32 * ((lens[b] - 1) // 32)  # whole blocks: their keys are there
        rows = at // 32
        ref, tol = _reference(k[:lens[b]], v[:lens[b]], q[:rows])
        assert np.all(np.abs(out[b, :rows] - ref) <= tol), b
    assert sd.get_device_error() == 0
