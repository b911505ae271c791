"""Attention over the 8-bit cache with even shares of a batch's keys for every SM: parts of
heads that a share's border cuts, joined from a workspace, against the float64 oracle."""
import numpy as np
import pytest
import torch

from paper_2606_31160_gb300 import sd
from tests.helpers import ensure_lib
from tests.test_gpu_kv8 import _attention_ok, _bf16, _cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_lib()
    sd.get_device_error()


def _workspace(q, c):
    """NaN throughout: nothing of it may count that was not written by the call."""
    B, R, Hq, D = q.shape
    need = sd.kv8_attention_workspace_bytes(B, R, Hq, c.shape[1], D, c.shape[2])
    assert need > 0  # even shares are taken
    return torch.full((need // 4,), float("nan"), dtype=torch.float32, device="cuda")


# whole heads and parts of them in a share; rows of one tile and of two; a head's first
# keys, a share's last and a scene's last anywhere in a tile
@pytest.mark.parametrize("D,block,cap,R,Hq,Hkv,B,shortest", [
    (128, 64, 1700, 9, 32, 8, 20, 9),
    (128, 32, 1633, 1, 21, 3, 54, 1),
    (64, 64, 2050, 6, 28, 4, 40, 6),
    (64, 128, 1800, 15, 16, 4, 39, 1500),
    (128, 128, 4200, 3, 4, 1, 78, 4000),
    (128, 64, 1600, 33, 9, 3, 18, 33),
])
@pytest.mark.parametrize("block_mask", [False, True])
def test_parity(D, block, cap, R, Hq, Hkv, B, shortest, block_mask):
    rng = np.random.default_rng(cap + B)
    lens = rng.integers(shortest, cap + 1, B).tolist()
    lens[0], lens[-1] = cap, shortest
    c = _cache(rng, B, Hkv, cap, D, block, lens=lens)
    for b, n in enumerate(lens):  # stale rows and the scales of blocks past the length
        c.k.view(torch.uint8)[b, :, n:] = 0x7f
        c.v.view(torch.uint8)[b, :, n:] = 0xff
        c.k_scale[b, :, -(-n // block):] = float("nan")
        c.v_scale[b, :, -(-n // block):] = float("inf")
    q = _bf16(rng.standard_normal((B, R, Hq, D)))
    out = torch.full_like(q, float("nan"))
    _attention_ok(sd.kv8_attention(q, c, out=out, block=block_mask, ws=_workspace(q, c)), q, c, block_mask)


def test_fewer_tiles_than_shares():
    """Lengths far below the capacity: most shares are empty."""
    rng = np.random.default_rng(3)
    B, cap = 78, 4200
    lens = rng.integers(2, 300, B).tolist()
    c = _cache(rng, B, 1, cap, 128, 64, lens=lens)
    q = _bf16(rng.standard_normal((B, 2, 4, 128)))
    _attention_ok(sd.kv8_attention(q, c, ws=_workspace(q, c)), q, c)


def test_scores_far_apart_over_the_parts():
    """The largest scores early, then late in the keys: the parts' references differ widely."""
    rng = np.random.default_rng(4)
    B, cap = 40, 1700
    c = _cache(rng, B, 4, cap, 128, 64, lens=rng.integers(1200, cap + 1, B).tolist())
    q = _bf16(rng.standard_normal((B, 7, 8, 128)) * 8)
    c.k_scale.copy_(c.k_scale * torch.linspace(0.02, 2.0, c.k_scale.shape[-1], device="cuda"))
    _attention_ok(sd.kv8_attention(q, c, ws=_workspace(q, c)), q, c)
    c.k_scale.copy_(c.k_scale.flip(-1))
    _attention_ok(sd.kv8_attention(q, c, ws=_workspace(q, c)), q, c)


def test_bad_lengths():
    rng = np.random.default_rng(5)
    B, cap = 40, 1700
    lens = rng.integers(5, 300, B).tolist()
    bad = {0: 4, 1: cap + 1, 17: -3, 33: 0, 34: 2 ** 30, B - 1: 3}
    for b, n in bad.items():
        lens[b] = n
    c = _cache(rng, B, 4, cap, 128, 64, lens=lens)
    q = _bf16(rng.standard_normal((B, 5, 8, 128)))
    out = torch.full_like(q, 3.0)
    sd.kv8_attention(q, c, out=out, ws=_workspace(q, c))
    assert sd.get_device_error() == sd.SD_DEVERR_LENGTH
    good = [b for b in range(B) if b not in bad]
    assert (out[list(bad)] == 3.0).all()
    part = sd.KV8Cache(c.k[good].contiguous(), c.v[good].contiguous(), c.k_scale[good].contiguous(),
                       c.v_scale[good].contiguous(), c.len[good].contiguous(), c.block)
    _attention_ok(out[good], q[good].contiguous(), part)
    c.len.fill_(cap + 1)  # no tile at all
    out.fill_(3.0)
    sd.kv8_attention(q, c, out=out, ws=_workspace(q, c))
    assert sd.get_device_error() == sd.SD_DEVERR_LENGTH and (out == 3.0).all()


def test_same_from_run_to_run_and_near_the_clusters():
    rng = np.random.default_rng(6)
    B, cap = 20, 3000
    c = _cache(rng, B, 8, cap, 128, 64, lens=rng.integers(2000, cap + 1, B).tolist())
    q = _bf16(rng.standard_normal((B, 8, 32, 128)))
    ws = _workspace(q, c)
    first = sd.kv8_attention(q, c, ws=ws).clone()
    for _ in range(3):
        assert torch.equal(sd.kv8_attention(q, c, ws=ws), first)
    assert torch.equal(sd.kv8_attention(q, c), first)
    sd.set_cluster_size(1)
    try:
        other = sd.kv8_attention(q, c)
    finally:
        sd.set_cluster_size(0)
    # sums in another order, then one rounding to bf16
    assert torch.allclose(other.float(), first.float(), rtol=2.0 ** -7, atol=2.0 ** -10)
    assert sd.get_device_error() == 0


def test_two_streams_and_a_graph():
    rng = np.random.default_rng(7)
    B, cap = 78, 1700
    c = _cache(rng, B, 4, cap, 64, 32, lens=rng.integers(300, cap + 1, B).tolist())
    q = _bf16(rng.standard_normal((B, 4, 16, 64)))
    want = sd.kv8_attention(q, c).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = [torch.empty_like(q) for _ in range(4)]
    for i, o in enumerate(outs):
        with torch.cuda.stream(side if i & 1 else torch.cuda.current_stream()):
            sd.kv8_attention(q, c, out=o)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sd.kv8_attention(q, c, out=outs[0])
    outs[0].zero_()
    g.replay()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want)


def test_workspace_refusals():
    rng = np.random.default_rng(8)
    c = _cache(rng, 40, 4, 1700, 128, 64, lens=[600] * 40)
    q = _bf16(rng.standard_normal((40, 4, 16, 128)))
    ws = _workspace(q, c)
    with pytest.raises(sd.SDError, match="WORKSPACE"):
        sd.kv8_attention(q, c, ws=ws[:-4])
    with pytest.raises(sd.SDError, match="INVALID_ARG"):
        sd.kv8_attention(q, c, ws=torch.empty(ws.numel() + 1, device="cuda")[1:])
    assert sd.kv8_attention_workspace_bytes(1, 4, 16, 4, 128, 600) == 0
    assert sd.kv8_attention_workspace_bytes(40, 4, 16, 3, 128, 1700) == 0
