"""Key weights with even shares of a batch's keys for every SM: row sums of runs from one
kernel, joined by the next, against the float64 oracle."""
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


def _bf16(x):
    return workloads.to_bf16(np.asarray(x, dtype=np.float32)).cuda()


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _workspace(q, cache):
    """NaN throughout: nothing of it may count that was not written by the call."""
    B, R, Hq, D = q.shape
    need = sd.attention_weights_workspace_bytes(B, R, Hq, cache.shape[1], D, cache.shape[2])
    assert need > 0  # even shares are taken
    return torch.full((need // 4,), float("nan"), dtype=torch.float32, device="cuda")


def _ok(got, ref, q, k, lens, rows):
    """The bound of the clusters' kernel: fp32 scores, an error of a few 2^-23 of the largest
    |q k| sqrt(D), which is as many parts in one of a weight; then sums of `rows` weights."""
    q, k = np.abs(to64(q)), np.abs(np.nan_to_num(to64(k)))
    for b, n in enumerate(lens):
        want = ref[b][:, :n]
        big = 2.0 ** -21 * q[b].max() * k[b].max() * np.sqrt(q.shape[-1])
        tol = (1e-5 + min(big, 1e-3)) * want + 1e-7 * rows
        assert np.all(np.abs(to64(got[b, :, :n]) - want) <= tol)


@pytest.mark.parametrize("D,cap,R,Hq,Hkv,B,shortest", [
    (128, 3000, 16, 32, 8, 12, 2000),
    (128, 2900, 32, 32, 8, 12, 32),
    (64, 4111, 11, 21, 3, 36, 11),
    (64, 2400, 33, 8, 4, 25, 2300),
])
@pytest.mark.parametrize("committed", [False, True])
def test_parity(D, cap, R, Hq, Hkv, B, shortest, committed):
    rng = np.random.default_rng(cap + R)
    lens = rng.integers(shortest, cap + 1, B).tolist()
    lens[0], lens[-1] = cap, shortest
    com = rng.integers(0, R + 1, B).tolist() if committed else None
    if com:
        com[1] = 0
    k = _bf16(rng.standard_normal((B, Hkv, cap, D)))
    for b, n in enumerate(lens):  # stale rows
        k[b, :, n:] = float("nan")
    q = _bf16(rng.standard_normal((B, R, Hq, D)))
    before = torch.from_numpy(rng.random((B, Hkv, cap)).astype(np.float32)).cuda() if committed else None
    out = torch.full((B, Hkv, cap), -3.0, device="cuda")
    cache = sd.KVCache(k, k, _i32(lens))
    sd.attention_weights(q, cache, before, out, 0.9, None if com is None else _i32(com), ws=_workspace(q, cache))
    assert sd.get_device_error() == 0
    ref = oracle.attention_weights(to64(q), np.nan_to_num(to64(k)), lens, com, None if before is None else to64(before), 0.9)
    _ok(out, ref, q, k, lens, R * Hq // Hkv)
    for b, n in enumerate(lens):
        assert (out[b, :, n:] == -3.0).all()


def test_fewer_tiles_than_shares_and_bad_scenes():
    rng = np.random.default_rng(2)
    B, R, cap = 12, 16, 3000
    lens = rng.integers(16, 200, B).tolist()
    com = rng.integers(0, R + 1, B).tolist()
    lens[0], lens[5], lens[11], com[7], com[8] = 15, cap + 1, -4, R + 1, -1
    bad = [0, 5, 7, 8, 11]
    k = _bf16(rng.standard_normal((B, 8, cap, 128)))
    q = _bf16(rng.standard_normal((B, R, 32, 128)))
    out = torch.full((B, 8, cap), -3.0, device="cuda")
    cache = sd.KVCache(k, k, _i32(lens))
    ws = _workspace(q, cache)
    sd.attention_weights(q, cache, weights=out, committed=_i32(com), ws=ws)
    assert sd.get_device_error() == sd.SD_DEVERR_LENGTH | sd.SD_DEVERR_ROLLBACK
    assert (out[bad] == -3.0).all()
    good = [b for b in range(B) if b not in bad]
    glens = [lens[b] for b in good]
    ref = oracle.attention_weights(to64(q[good]), to64(k[good][:, :, :256]), glens, [com[b] for b in good])
    _ok(out[good], ref, q[good], k[good][:, :, :256], glens, R * 4)
    cache.len.fill_(0)  # no tile at all
    out.fill_(-3.0)
    sd.attention_weights(q, cache, weights=out, ws=ws)
    assert sd.get_device_error() == sd.SD_DEVERR_LENGTH and (out == -3.0).all()


def test_in_place_repeats_streams_and_a_graph():
    rng = np.random.default_rng(3)
    B, R, cap = 12, 16, 3000
    lens = rng.integers(2000, cap + 1, B).tolist()
    k = _bf16(rng.standard_normal((B, 8, cap, 128)))
    q = _bf16(rng.standard_normal((B, R, 32, 128)))
    cache = sd.KVCache(k, k, _i32(lens))
    ws = _workspace(q, cache)
    first = sd.attention_weights(q, cache, ws=ws).clone()
    assert torch.equal(sd.attention_weights(q, cache, ws=ws), first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = [torch.zeros_like(first) for _ in range(4)]
    for i, o in enumerate(outs):
        with torch.cuda.stream(side if i & 1 else torch.cuda.current_stream()):
            sd.attention_weights(q, cache, weights=o)
    torch.cuda.synchronize()
    assert all(torch.equal(o, first) for o in outs)
    acc = first.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sd.attention_weights(q, cache, weights_in=acc, weights=acc, decay=0.5)
    g.replay()
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        old = n - R  # a key of the pass has no weight from before
        assert torch.allclose(acc[b, :, :old], 1.5 * first[b, :, :old], rtol=1e-6, atol=0)
        assert torch.equal(acc[b, :, old:n], first[b, :, old:n])
    sd.set_cluster_size(2)
    try:
        other = sd.attention_weights(q, cache)
    finally:
        sd.set_cluster_size(0)
    assert torch.allclose(other, first, rtol=1e-3, atol=1e-7 * R * 4)
    assert sd.get_device_error() == 0


def test_workspace_refusals():
    k = torch.zeros((12, 8, 3000, 128), dtype=torch.bfloat16, device="cuda")
    cache = sd.KVCache(k, k, _i32([3000] * 12))
    q = torch.zeros((12, 16, 32, 128), dtype=torch.bfloat16, device="cuda")
    ws = _workspace(q, cache)
    with pytest.raises(sd.SDError, match="WORKSPACE"):
        sd.attention_weights(q, cache, ws=ws[:-4])
    with pytest.raises(sd.SDError, match="INVALID_ARG"):
        sd.attention_weights(q, cache, ws=torch.empty(ws.numel() + 1, device="cuda")[1:])
    assert sd.attention_weights_workspace_bytes(1, 16, 32, 8, 128, 3000) == 0
    assert sd.attention_weights_workspace_bytes(12, 40, 32, 8, 128, 3000) == 0  # more than 128 rows
