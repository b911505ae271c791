"""Appending to a paged cache and committing what a tree's acceptance kept, against the
float64 oracle. Rows that only move are compared bit for bit; a rotated element x of a
pair may be off by half a bf16 step of the exact value and by the rotation's fp32
error (helpers.rope_bound)."""
import numpy as np
import pytest
import torch

import oracle
from helpers import pair_magnitude, rope_bound, to64
from paper_2606_31160_gb300 import build, sd

pytestmark = pytest.mark.gpu

SECTIONS = {128: (16, 24, 24), 64: (8, 12, 12)}


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    sd.get_device_error()


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)


def make_cache(g, lens, cap, Hkv, D, page, spare=3):
    """A cache with random rows, its pages in a random order; what no scene owns is NaN."""
    B, per = len(lens), -(-cap // page)
    n = B * per + spare
    table = torch.randperm(n, generator=g, device="cuda")[:B * per].view(B, per).to(torch.int32)
    k, v = _randn(g, n, Hkv, page, D), _randn(g, n, Hkv, page, D)
    free = torch.ones(n, dtype=torch.bool, device="cuda")
    free[table.flatten().long()] = False
    k[free], v[free] = float("nan"), float("nan")
    return sd.PagedKVCache(k, v, table, _i32(lens))


def rows_of(cache, b, n, which="k"):
    """[n, Hkv, D] float64"""
    pool = to64(getattr(cache, which))
    return np.swapaxes(oracle.gather_pages(pool, cache.table[b].cpu().numpy(), n), 0, 1)


@pytest.mark.parametrize("B,R,Hq,Hkv,D,page,interleaved,fused,ragged", [
    (1, 1, 4, 1, 64, 16, 0, False, False),
    (1, 8, 32, 8, 128, 64, 0, True, False),
    (3, 21, 28, 4, 64, 16, 1, False, True),
    (2, 130, 8, 8, 128, 128, 0, True, True),
    (5, 17, 7, 1, 128, 32, 1, True, True),
    (2, 300, 16, 4, 64, 32, 0, True, False),
])
def test_append(B, R, Hq, Hkv, D, page, interleaved, fused, ragged):
    g = torch.Generator(device="cuda").manual_seed(B * 1000 + R)
    rng = np.random.default_rng(R)
    lens = rng.integers(0, 90, B)
    lens[0] = page - 1 if R > 1 else 0  # the rows cross a page's end
    cache = make_cache(g, lens, 90 + R, Hkv, D, page)
    n_new = rng.integers(0, R + 1, B) if ragged else np.full(B, R)
    pos = rng.integers(0, 1 << 20, (B, R, 3))
    if fused:
        q, k, v = _randn(g, B, R, Hq + 2 * Hkv, D).split([Hq, Hkv, Hkv], dim=2)
    else:
        q, k, v = _randn(g, B, R, Hq, D), _randn(g, B, R, Hkv, D), _randn(g, B, R, Hkv, D)
    q0, k0, v0 = q.clone(), k.clone(), v.clone()
    pool_k, pool_v = cache.k.clone(), cache.v.clone()
    q_out = torch.full((B, R, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    got = sd.paged_append(cache, k, v, q=q, pos=_i32(pos), sections=SECTIONS[D], interleaved=interleaved, base=1e6,
                          n_new=_i32(n_new) if ragged else None, q_out=q_out)
    assert got is q_out and sd.get_device_error() == 0
    assert torch.equal(q, q0) and torch.equal(k, k0) and torch.equal(v, v0)
    assert cache.len.tolist() == (lens + n_new).tolist()
    written = torch.zeros(pool_k.shape[:3], dtype=torch.bool, device="cuda")
    for b in range(B):
        n = int(n_new[b])
        at = int(lens[b]) + np.arange(n)
        pages = cache.table[b].cpu().numpy()[at // page]
        written[pages, :, at % page] = True
        for x, out in ((q0, q_out[b, :n]), (k0, cache.k[pages, :, at % page])):
            x64 = to64(x[b, :n])
            want = oracle.mrope_apply(x64, pos[b, :n, None], SECTIONS[D], interleaved, 1e6)
            assert np.all(np.abs(to64(out) - want) <= rope_bound(want, pair_magnitude(x64)))
        assert torch.equal(cache.v[pages, :, at % page], v0[b, :n])
        assert (q_out[b, n:] == 7.0).all()
    # nothing else was touched
    keep = ~written
    assert torch.equal(cache.k[keep].view(torch.int16), pool_k[keep].view(torch.int16))
    assert torch.equal(cache.v[keep].view(torch.int16), pool_v[keep].view(torch.int16))


@pytest.mark.parametrize("R", [5, 700])
def test_append_is_the_rotation_and_the_append(R):
    """Bit for bit what sd.rope_apply gives, in place and strided; without positions a copy."""
    g = torch.Generator(device="cuda").manual_seed(1)
    B, Hq, Hkv, D = 2, 8, 2, 128
    pos = torch.randint(0, 5000, (B, R, 3), generator=g, device="cuda", dtype=torch.int32)
    qkv = _randn(g, B, R, Hq + 2 * Hkv, D)
    q, k, v = qkv.split([Hq, Hkv, Hkv], dim=2)
    q1, k1 = q.contiguous(), k.contiguous()
    sd.rope_apply(q1, k1, pos, SECTIONS[D])
    cache = make_cache(g, [3, 40], 40 + R, Hkv, D, 16)
    sd.paged_append(cache, k, v, q=q, pos=pos, sections=SECTIONS[D])
    assert torch.equal(q, q1) and torch.equal(k, qkv[:, :, Hq:Hq + Hkv])
    for b, n0 in ((0, 3), (1, 40)):
        assert np.array_equal(rows_of(cache, b, n0 + R)[n0:], to64(k1[b]))
        assert np.array_equal(rows_of(cache, b, n0 + R, "v")[n0:], to64(v[b]))
    plain = make_cache(g, [3, 40], 40 + R, Hkv, D, 16)
    sd.paged_append(plain, k, v)
    assert np.array_equal(rows_of(plain, 0, 3 + R)[3:], to64(k[0]))
    assert sd.get_device_error() == 0


def test_append_errors_leave_the_scene():
    g = torch.Generator(device="cuda").manual_seed(2)
    B, R, Hq, Hkv, D, page = 4, 6, 4, 2, 64, 16
    sec = SECTIONS[D]
    pos = torch.zeros((B, R, 3), dtype=torch.int32, device="cuda") + 9

    def check(bit, lens, n_new=None, bad_page=None, good=(0, 2, 3)):
        cache = make_cache(g, lens, 48, Hkv, D, page)
        if bad_page is not None:
            cache.table[1, bad_page[0]] = bad_page[1]
        q, k, v = _randn(g, B, R, Hq, D), _randn(g, B, R, Hkv, D), _randn(g, B, R, Hkv, D)
        q0, pool = q.clone(), cache.k.clone()
        own = cache.table[1].clone()
        sd.paged_append(cache, k, v, q=q, pos=pos, sections=sec, n_new=None if n_new is None else _i32(n_new))
        assert sd.get_device_error() == bit
        assert cache.len[1] == lens[1] and torch.equal(q[1], q0[1])
        own = own[(own >= 0) & (own < pool.shape[0])].long()
        assert torch.equal(cache.k[own].view(torch.int16), pool[own].view(torch.int16))
        for b in good:
            assert cache.len[b] == lens[b] + (R if n_new is None else n_new[b])
            if n_new is None or n_new[b]:
                assert not torch.equal(q[b], q0[b])

    check(sd.SD_DEVERR_KV_OVERFLOW, [3, 43, 5, 42])
    check(sd.SD_DEVERR_LENGTH, [3, -1, 5, 42])
    check(sd.SD_DEVERR_LENGTH, [3, 7, 5, 42], n_new=[6, 7, 0, 2])
    check(sd.SD_DEVERR_LENGTH, [3, 7, 5, 42], n_new=[6, -1, 0, 2])
    for entry in (-1, 1 << 30, -(1 << 31)):
        check(sd.SD_DEVERR_PAGE, [3, 14, 5, 42], bad_page=(1, entry))
    # an entry that no new row needs may be anything
    cache = make_cache(g, [3, 14, 5, 42], 48, Hkv, D, page)
    cache.table[1, 2] = -1
    sd.paged_append(cache, _randn(g, B, R, Hkv, D), _randn(g, B, R, Hkv, D))
    assert sd.get_device_error() == 0


def _path(rng, n):
    m = int(rng.integers(0, n + 1))
    return np.sort(rng.choice(n, m, replace=False)) if m else np.zeros(0, dtype=np.int64)


@pytest.mark.parametrize("B,R,Hkv,D,page,layers,ragged", [
    (1, 1, 1, 64, 16, 1, False),
    (1, 26, 8, 128, 64, 36, False),
    (6, 61, 4, 64, 16, 3, True),
    (3, 256, 2, 128, 32, 2, True),
    (2, 9, 3, 128, 128, 50, False),
    (2, 700, 2, 64, 64, 2, True),
])
def test_commit(B, R, Hkv, D, page, layers, ragged):
    g = torch.Generator(device="cuda").manual_seed(R)
    rng = np.random.default_rng(B + R)
    n_new = rng.integers(0, R + 1, B) if ragged else np.full(B, R)
    lens = rng.integers(0, 70, B) + n_new
    shape = [make_cache(g, lens, 70 + R, Hkv, D, page) for _ in range(layers)]
    paths = [_path(rng, int(n)) for n in n_new]
    paths[0] = np.arange(0, n_new[0], 2)  # rows that others move over
    path = np.full((B, R), 1 << 30)
    for b, p in enumerate(paths):
        path[b, :len(p)] = p
    before = [(c.k.clone(), c.v.clone()) for c in shape]
    sd.paged_commit(shape, _i32(path), _i32([len(p) for p in paths]), n_new=_i32(n_new) if ragged else None)
    assert sd.get_device_error() == 0
    for c, pools in zip(shape, before):
        first = lens - n_new
        assert c.len.tolist() == [int(f) + len(p) for f, p in zip(first, paths)]
        for which, old in (("k", pools[0]), ("v", pools[1])):
            moved = old.clone()
            for b, p in enumerate(paths):
                t = c.table[b].cpu().numpy()
                src, dst = first[b] + p, first[b] + np.arange(len(p))
                moved[t[dst // page], :, dst % page] = old[t[src // page], :, src % page]
            assert torch.equal(getattr(c, which).view(torch.int16), moved.view(torch.int16))


def test_commit_errors_leave_the_scene():
    g = torch.Generator(device="cuda").manual_seed(3)
    good = [0, 2, 5, -1, -1, -1]
    for bit, lens, n_new, path, emit, entry in (
            (sd.SD_DEVERR_ROLLBACK, 20, 6, [0, 2, 2, 0, 0, 0], 3, None), (sd.SD_DEVERR_ROLLBACK, 20, 6, [0, 3, 2, 0, 0, 0], 3, None),
            (sd.SD_DEVERR_ROLLBACK, 20, 6, [0, 2, 6, 0, 0, 0], 3, None), (sd.SD_DEVERR_ROLLBACK, 20, 6, [-1, 2, 3, 0, 0, 0], 3, None),
            (sd.SD_DEVERR_ROLLBACK, 20, 6, [0, 1 << 30, 3, 0, 0, 0], 2, None), (sd.SD_DEVERR_ROLLBACK, 20, 4, good, 3, None),
            (sd.SD_DEVERR_ROLLBACK, 20, 6, good, 7, None), (sd.SD_DEVERR_ROLLBACK, 20, 6, good, -1, None),
            (sd.SD_DEVERR_LENGTH, 5, 6, good, 3, None), (sd.SD_DEVERR_LENGTH, 65, 6, good, 3, None),
            (sd.SD_DEVERR_LENGTH, 20, 7, good, 3, None), (sd.SD_DEVERR_LENGTH, 20, -1, good, 3, None),
            (sd.SD_DEVERR_PAGE, 20, 6, good, 3, -1), (sd.SD_DEVERR_PAGE, 20, 6, good, 3, 1 << 20)):
        cache = make_cache(g, [30, lens], 64, 2, 64, 16)
        if entry is not None:
            cache.table[1, 1] = entry
        k = cache.k.clone()
        sd.paged_commit(cache, _i32([good, path]), _i32([3, emit]), n_new=_i32([6, n_new]))
        assert sd.get_device_error() == bit, (bit, lens, n_new, path, emit)
        assert cache.len.tolist() == [27, lens]
        own = cache.table[1][(cache.table[1] >= 0) & (cache.table[1] < k.shape[0])].long()
        assert torch.equal(cache.k[own].view(torch.int16), k[own].view(torch.int16))
    # n_emit 0 drops all the new rows; a table entry that no kept row needs may be anything
    cache = make_cache(g, [30, 20], 64, 2, 64, 16)
    cache.table[1, 2:] = -1
    sd.paged_commit([cache], _i32([good, good]), _i32([0, 1]), n_new=_i32([6, 6]))
    assert sd.get_device_error() == 0 and cache.len.tolist() == [24, 15]


def test_rows_past_32_bits_of_elements():
    """A pool of more than 2^32 elements: its last pages, by append and commit."""
    Hkv, page, D = 8, 128, 128
    n = (1 << 32) // (Hkv * page * D) + 5
    k, v = (torch.zeros((n, Hkv, page, D), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    g = torch.Generator(device="cuda").manual_seed(4)
    table = _i32([[n - 1, n - 3], [n - 2, 0]])
    cache = sd.PagedKVCache(k, v, table, _i32([126, 127]))
    kn, vn = _randn(g, 2, 4, Hkv, D), _randn(g, 2, 4, Hkv, D)
    sd.paged_append(cache, kn, vn)
    assert torch.equal(k[n - 1, :, 126:], kn[0, :2].transpose(0, 1)) and torch.equal(v[n - 3, :, :2], vn[0, 2:].transpose(0, 1))
    assert torch.equal(k[n - 2, :, 127], kn[1, 0]) and torch.equal(v[0, :, :3], vn[1, 1:].transpose(0, 1))
    sd.paged_commit(cache, _i32([[1, 3, -1, -1], [0, 3, -1, -1]]), _i32([2, 2]))
    assert torch.equal(k[n - 1, :, 126:], kn[0, [1, 3]].transpose(0, 1)) and torch.equal(v[0, :, 0], vn[1, 3])
    assert sd.get_device_error() == 0
