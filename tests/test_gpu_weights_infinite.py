"""Key weights where a score is infinite: a key at -inf has weight 0 and the others are
what they are without it, wherever it lies; a row with a score of +inf has none (NaN)."""
import numpy as np
import pytest
import torch

import oracle
from paper_2606_31160_gb300 import sd, workloads
from tests.helpers import ensure_lib, to64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_lib()
    sd.get_device_error()
    yield
    sd.set_cluster_size(0)


def _inputs(B, n, R, Hq, Hkv, D):
    """Every query's element 5 is positive."""
    rng = np.random.default_rng(n + R)
    k = workloads.to_bf16(rng.standard_normal((B, Hkv, n, D)).astype(np.float32))
    q = rng.standard_normal((B, R, Hq, D))
    q[..., 5] = np.abs(q[..., 5]) + 0.5
    return k, workloads.to_bf16(q.astype(np.float32))


SHAPES = [(1, 700, 3, 4, 2, 128), (1, 2500, 8, 16, 4, 64), (1, 900, 12, 8, 2, 128), (1, 1500, 30, 8, 2, 128),
          (1, 700, 70, 4, 1, 64), (12, 1800, 16, 32, 8, 128)]


@pytest.mark.parametrize("B,n,R,Hq,Hkv,D", SHAPES)
@pytest.mark.parametrize("cs", [0, 1, 4])
def test_keys_at_minus_infinity(B, n, R, Hq, Hkv, D, cs):
    k, q = _inputs(B, n, R, Hq, Hkv, D)
    at = [0, 1, 37, 127, 128, 300, n - R]
    k[:, :, at, 5] = -float("inf")
    cache = sd.KVCache(k.cuda(), k.cuda(), torch.full((B,), n, dtype=torch.int32, device="cuda"))
    sd.set_cluster_size(cs)
    try:
        got = to64(sd.attention_weights(q.cuda(), cache))
    finally:
        sd.set_cluster_size(0)
    ref = oracle.attention_weights(to64(q), to64(k), [n] * B)
    assert (got[:, :, at] == 0).all()
    # fp32: a few roundings of a score, sums of positive terms
    assert np.all(np.abs(got - ref) <= 2e-5 * ref + 1e-6 * R * Hq / Hkv)
    assert sd.get_device_error() == 0


@pytest.mark.parametrize("B,n,R,Hq,Hkv,D", SHAPES[:-1])
@pytest.mark.parametrize("at", [0, 200])
def test_a_key_at_plus_infinity(B, n, R, Hq, Hkv, D, at):
    k, q = _inputs(B, n, R, Hq, Hkv, D)
    k[:, 0, at, 5] = float("inf")
    cache = sd.KVCache(k.cuda(), k.cuda(), torch.full((B,), n, dtype=torch.int32, device="cuda"))
    got = sd.attention_weights(q.cuda(), cache)
    assert got[:, 0].isnan().all() and not got[:, 1:].isnan().any()
    assert sd.get_device_error() == 0
