"""A key that is no number makes the rows that see it NaN, wherever it lies: alone in its
tile or its part of the keys, or far below the other keys of its row."""
import numpy as np
import pytest
import torch

import oracle
from paper_2606_31160_gb300 import sd, workloads
from tests.helpers import ensure_lib

pytestmark = pytest.mark.gpu

NAN = 0x7f


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_lib()
    sd.get_device_error()
    yield
    sd.set_cluster_size(0)


def _cache(rng, B, H, n, D):
    c = sd.KV8Cache.empty(B, H, n, D, 64)
    for t in (c.k, c.v):
        x = oracle.round_e4m3(np.clip(rng.standard_normal((B, H, n, D)) * 100, -448, 448))
        t.copy_(torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).cuda())
    c.k_scale.fill_(2.0 ** -7)
    c.v_scale.fill_(2.0 ** -7)
    c.len.fill_(n)
    return c


def _queries(rng, *shape):
    return workloads.to_bf16(rng.standard_normal(shape).astype(np.float32)).cuda()


def _nan_rows_only(out, good, head, G, from_row=0):
    """Head `head`'s rows from from_row on are NaN; the rest is what it was."""
    want = torch.zeros(out.shape[:3], dtype=torch.bool, device="cuda")
    want[:, from_row:, head * G:(head + 1) * G] = True
    assert out[want].isnan().all(), int((~out[want].isnan()).sum())
    assert torch.equal(out[~want], good[~want])


@pytest.mark.parametrize("cs", [0, 1, 2, 4, 8, 16])
@pytest.mark.parametrize("D", [64, 128])
def test_alone_in_its_tile(D, cs):
    """The newest key, the only one of its tile, in the tiles of either softmax group and in
    the last CTA's range; with R = 3 under the block mask the three newest."""
    rng = np.random.default_rng(D + cs)
    sd.set_cluster_size(cs)
    try:
        for n, R, block in ((129, 1, False), (257, 1, False), (1281, 1, True), (131, 3, True), (1665, 1, False)):
            c = _cache(rng, 1, 3, n, D)
            q = _queries(rng, 1, R, 12, D)
            good = sd.kv8_attention(q, c, block=block).clone()
            c.k.view(torch.uint8)[0, 1, n - R:, 9] = NAN
            _nan_rows_only(sd.kv8_attention(q, c, block=block), good, 1, 4)
    finally:
        sd.set_cluster_size(0)
    assert sd.get_device_error() == 0


def test_the_rows_that_see_it():
    """The last new key, alone in its tile: the last row sees it."""
    rng = np.random.default_rng(1)
    c = _cache(rng, 1, 2, 257, 128)
    q = _queries(rng, 1, 5, 8, 128)
    good = sd.kv8_attention(q, c).clone()
    c.k.view(torch.uint8)[0, 0, 256, 3] = NAN
    _nan_rows_only(sd.kv8_attention(q, c), good, 0, 4, from_row=4)


@pytest.mark.parametrize("tile", [0, 1, 6, 7])
def test_a_whole_tile(tile):
    rng = np.random.default_rng(2)
    for cs in (1, 2, 4, 8):
        sd.set_cluster_size(cs)
        try:
            c = _cache(rng, 1, 2, 1024, 64)
            q = _queries(rng, 1, 2, 6, 64)
            good = sd.kv8_attention(q, c).clone()
            c.k.view(torch.uint8)[0, 1, 128 * tile:128 * tile + 126, 0] = NAN
            _nan_rows_only(sd.kv8_attention(q, c), good, 1, 3)
        finally:
            sd.set_cluster_size(0)


@pytest.mark.parametrize("cs", [0, 1, 2])
def test_far_below_the_rest(cs):
    """Beside finite keys whose scores lie hundreds below another tile's."""
    rng = np.random.default_rng(3)
    sd.set_cluster_size(cs)
    try:
        for tile, at in ((1, 40), (0, 200)):
            c = _cache(rng, 1, 2, 256, 128)
            c.k.view(torch.uint8)[:, :, 128 * tile:128 * (tile + 1)] = 0x7e  # 448 in every place
            q = (_queries(rng, 1, 1, 8, 128).abs() + 4.0).contiguous()
            good = sd.kv8_attention(q, c).clone()
            c.k.view(torch.uint8)[0, 0, at, 5] = NAN
            _nan_rows_only(sd.kv8_attention(q, c), good, 0, 4)
    finally:
        sd.set_cluster_size(0)


def test_even_shares():
    """Parts of heads that a share's border cuts: the newest key of every third scene."""
    rng = np.random.default_rng(4)
    B, cap, D = 78, 4225, 128
    c = _cache(rng, 1, 1, cap, D)
    k, v = (t.view(torch.uint8).expand(B, -1, -1, -1).contiguous().view(torch.float8_e4m3fn) for t in (c.k, c.v))
    lens = 128 * rng.integers(29, 34, B) + 1
    c = sd.KV8Cache(k, v, c.k_scale.expand(B, -1, -1).contiguous(), c.v_scale.expand(B, -1, -1).contiguous(),
                    torch.from_numpy(lens.astype(np.int32)).cuda(), 64)
    q = _queries(rng, B, 1, 4, D)
    assert sd.kv8_attention_workspace_bytes(B, 1, 4, 1, D, cap) > 0
    good = sd.kv8_attention(q, c).clone()
    assert not good.isnan().any()
    bad = torch.zeros(B, dtype=torch.bool, device="cuda")
    for b in range(0, B, 3):
        k.view(torch.uint8)[b, 0, lens[b] - 1, 7] = NAN
        bad[b] = True
    out = sd.kv8_attention(q, c)
    assert out[bad].isnan().all() and torch.equal(out[~bad], good[~bad])
    assert sd.get_device_error() == 0
