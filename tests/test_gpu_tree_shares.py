"""The tree attention in even shares (the way of large batches, whose cut units a second kernel
joins), for every number of packed rows and both head dims, against the float64 oracle. That a
shape is served in shares is checked by what such a call does without its workspace: it is
refused."""
import numpy as np
import pytest
import torch

from paper_2606_31160_gb300 import build, sd
from test_gpu_paged import _i32, _randn, make_cache
from test_gpu_tree import check_scene, make_tree, test_attention_of_many_scenes as many_scenes

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    sd.get_device_error()


def takes_shares(q, cache, **kw):
    try:
        sd.tree_attention(q, cache, ws=torch.empty(0, dtype=torch.uint8, device="cuda"), **kw)
    except sd.SDError as e:
        return e.status == sd.SD_ERR_WORKSPACE
    return False


# B, R, Hq, Hkv, D, L: the packed rows of a KV head (G R) up to 32, 64, 128 and past that
SHAPES = [(40, 6, 8, 4, 128, 1900), (20, 8, 32, 8, 128, 1900),            # 12, 32
          (40, 20, 8, 4, 128, 2000), (20, 9, 28, 4, 128, 4000),           # 40, 63
          (20, 26, 32, 8, 128, 2900), (80, 30, 8, 2, 128, 3000),          # 104, 120
          (40, 33, 16, 4, 128, 5000),                                     # 132
          (100, 5, 4, 2, 64, 3000), (20, 8, 32, 8, 64, 2900),             # 10, 32
          (80, 15, 8, 2, 64, 4000), (20, 16, 32, 8, 64, 2900),            # 60, 64
          (20, 26, 32, 8, 64, 2900), (40, 32, 16, 4, 64, 2900), (40, 13, 28, 4, 64, 2900),  # 104, 128, 91
          (42, 70, 8, 4, 64, 3500)]                                       # 140


@pytest.mark.parametrize("B,R,Hq,Hkv,D,L", SHAPES)
def test_shapes_are_served_in_shares(B, R, Hq, Hkv, D, L):
    """With the cache that the tests below make of them."""
    pool = torch.zeros((1, Hkv, 64, D), dtype=torch.bfloat16, device="cuda")
    cache = sd.PagedKVCache(pool, pool.clone(), torch.zeros((B, -(-(L + R) // 64)), dtype=torch.int32, device="cuda"),
                            torch.full((B,), R, dtype=torch.int32, device="cuda"))
    assert takes_shares(torch.zeros((B, R, Hq, D), dtype=torch.bfloat16, device="cuda"), cache)


@pytest.mark.parametrize("B,R,Hq,Hkv,D,L", [s for s in SHAPES if s not in ((100, 5, 4, 2, 64, 3000), (80, 15, 8, 2, 64, 4000),
                                                                          (80, 30, 8, 2, 128, 3000), (40, 33, 16, 4, 128, 5000),
                                                                          (42, 70, 8, 4, 64, 3500))])
def test_ragged_batches_in_shares(B, R, Hq, Hkv, D, L):
    """As test_gpu_tree's, which has the five left out here: trees, scenes with nothing new, some
    that are not valid, any workspace, the same bits again."""
    many_scenes(B, R, Hq, Hkv, D, L)


@pytest.mark.parametrize("B,R,Hq,Hkv,D,L", SHAPES)
def test_no_numbers_in_shares(B, R, Hq, Hkv, D, L):
    """Values and keys of new rows that are no numbers reach only the rows that see them, also
    where a share's border cuts the unit."""
    g = torch.Generator(device="cuda").manual_seed(R)
    rng = np.random.default_rng(R)
    lens = rng.integers(L // 2, L + 1, B) + R
    cache = make_cache(g, lens, L + R, Hkv, D, 64)
    parents = np.stack([make_tree(rng, R, forest=True) for _ in range(B)])
    for b in range(B):
        t, at = cache.table[b], int(lens[b]) - R
        for row, key, value in ((R - 1, float("nan"), 1.0), (R - 2, None, float("inf")), (R // 2, None, float("nan"))):
            n = at + row
            if key is not None:
                cache.k[t[n // 64], :, n % 64, 5] = key
            cache.v[t[n // 64], :, n % 64, 7] = value
    q = _randn(g, B, R, Hq, D)
    assert takes_shares(q, cache, parents=_i32(parents))
    out = sd.tree_attention(q, cache, parents=_i32(parents))
    assert sd.get_device_error() == 0
    for b in range(0, B, 3):
        check_scene(out, q, cache, b, parents[b], R)


WIDE = [(1, 1, 16, 4, 128, 300, 131072), (1, 9, 16, 4, 128, 2000, 131072), (2, 26, 32, 8, 128, 129, 65536),
        (3, 61, 16, 4, 128, 640, 65536), (2, 130, 8, 2, 128, 1500, 131072), (1, 5, 8, 4, 64, 1, 131072),
        (2, 13, 28, 4, 64, 777, 131072), (3, 40, 32, 4, 64, 513, 131072), (4, 12, 32, 8, 64, 128, 65536)]


@pytest.mark.parametrize("B,R,Hq,Hkv,D,keys,width", WIDE)
def test_tables_wider_than_the_keys(B, R, Hq, Hkv, D, keys, width):
    """A table as wide as a long context, with few keys in it. Most of these are served in shares,
    fewer tiles than CTAs, one a share, units of many parts; the others in clusters of which not
    every CTA has a tile. What lies past a scene's pages is anything."""
    g = torch.Generator(device="cuda").manual_seed(keys)
    rng = np.random.default_rng(keys)
    lens = rng.integers(0, keys + 1, B) + R
    lens[-1] = keys + R
    small = make_cache(g, lens, keys + R, Hkv, D, 64)
    table = torch.full((B, width // 64), -1, dtype=torch.int32, device="cuda")
    table[:, 1::2] = 1 << 30
    table[:, :small.table.shape[1]] = small.table
    cache = sd.PagedKVCache(small.k, small.v, table, small.len)
    parents = np.stack([make_tree(rng, R, forest=True) for _ in range(B)])
    q = _randn(g, B, R, Hq, D)
    ws = torch.full((sd.tree_attention_workspace_bytes(B, R, Hq, Hkv, D, width),), 0xFF, dtype=torch.uint8, device="cuda")
    out = sd.tree_attention(q, cache, parents=_i32(parents), ws=ws)
    assert sd.get_device_error() == 0
    for b in range(B):
        check_scene(out, q, cache, b, parents[b], R)


@pytest.mark.parametrize("D", [64, 128])
def test_wide_tables_are_served_in_shares(D):
    """Some of the shapes above, for each head dim."""
    def shares(B, R, Hq, Hkv, D, keys, width):
        pool = torch.zeros((1, Hkv, 64, D), dtype=torch.bfloat16, device="cuda")
        cache = sd.PagedKVCache(pool, pool.clone(), torch.zeros((B, width // 64), dtype=torch.int32, device="cuda"),
                                torch.full((B,), R, dtype=torch.int32, device="cuda"))
        return takes_shares(torch.zeros((B, R, Hq, D), dtype=torch.bfloat16, device="cuda"), cache)
    ways = [shares(*s) for s in WIDE if s[4] == D]
    assert sum(ways) >= 2
