"""Host checks of the paged cache and the tree calls: a bad argument returns its status
before anything is launched (no GPU needed), and the binding refuses what it can see."""
import ctypes

import pytest
import torch

from paper_2606_31160_gb300 import build, sd


@pytest.fixture(scope="module")
def lib():
    build.build()
    return sd.lib()


P = ctypes.c_void_p
SEC = (ctypes.c_int32 * 3)(16, 24, 24)


def _struct(k=16, v=16, table=16, n=16, ticket=16, B=1, H=8, n_pages=40, page=64, max_pages=4, D=128):
    return sd.PagedCacheStruct(k, v, table, n, ticket, B, H, n_pages, page, max_pages, D)


def _cache(**kw):
    return ctypes.byref(_struct(**kw))


BAD_CACHES = [(dict(k=0), 1), (dict(v=0), 1), (dict(table=0), 1), (dict(n=0), 1), (dict(ticket=0), 1), (dict(k=24), 1),
              (dict(H=0), 1), (dict(B=-1), 1), (dict(n_pages=0), 1), (dict(max_pages=0), 1), (dict(D=96), 2), (dict(page=48), 2),
              (dict(page=256), 2), (dict(page=8), 2), (dict(B=70000), 2), (dict(max_pages=1 << 25), 2), (dict(n_pages=1 << 29), 2),
              (dict(H=40000), 2)]


def _append(lib, c, k=16, ks=1024, v=16, vs=1024, q=16, qs=4096, qo=0, R=8, Hq=32, pos=16, sec=SEC, inter=0, base=1e6, n=0):
    return lib.sd_paged_append(c, P(k), ks, P(v), vs, P(q), qs, P(qo), R, Hq, P(pos), sec, inter, base, P(n), None)


def test_append(lib):
    assert _append(lib, None) == 1
    for kw, status in BAD_CACHES:
        assert _append(lib, _cache(**kw)) == status, kw
    c = _cache()
    assert _append(lib, c, k=0) == 1 and _append(lib, c, v=0) == 1 and _append(lib, c, k=8) == 1 and _append(lib, c, q=8) == 1
    assert _append(lib, c, q=0) == 1 and _append(lib, c, Hq=0) == 1             # queries and their heads go together
    assert _append(lib, c, q=0, Hq=0, qo=16) == 1 and _append(lib, c, qo=24) == 1
    assert _append(lib, c, pos=0) == 1                                          # queries to rotate, nowhere
    assert _append(lib, c, ks=1023) == 1 and _append(lib, c, ks=1028) == 1 and _append(lib, c, vs=512) == 1
    assert _append(lib, c, qs=4095) == 1 and _append(lib, c, qs=4100) == 1
    assert _append(lib, c, R=-1) == 1 and _append(lib, c, Hq=-1) == 1
    assert _append(lib, c, inter=2) == 1 and _append(lib, c, base=1.0) == 1 and _append(lib, c, sec=None) == 1
    assert _append(lib, c, sec=(ctypes.c_int32 * 3)(16, 24, 23)) == 1
    assert _append(lib, c, R=0) == 0 and _append(lib, _cache(B=0, k=0)) == 0


def _attend(lib, c, q=16, qs=4096, parents=0, n=0, out=16, R=8, Hq=32, scale=0.0, ws=16, nbytes=1 << 30):
    return lib.sd_tree_attention(P(q), qs, c, P(parents), P(n), P(out), R, Hq, scale, P(ws), nbytes, None)


def test_attention(lib):
    assert _attend(lib, None) == 1
    for kw, status in BAD_CACHES:
        assert _attend(lib, _cache(**kw)) == status, kw
    c = _cache()
    assert _attend(lib, c, R=0) == 1 and _attend(lib, c, Hq=30) == 1 and _attend(lib, c, Hq=0) == 1
    assert _attend(lib, c, R=257) == 2
    assert _attend(lib, c, scale=-1.0) == 1 and _attend(lib, c, scale=float("nan")) == 1 and _attend(lib, c, scale=float("inf")) == 1
    assert _attend(lib, c, scale=3e38) == 1                                     # past fp32 in the units of the exponent
    assert _attend(lib, c, qs=4088) == 1 and _attend(lib, c, qs=4097) == 1
    assert _attend(lib, c, q=0) == 1 and _attend(lib, c, out=0) == 1 and _attend(lib, c, q=8) == 1 and _attend(lib, c, out=8) == 1
    assert _attend(lib, c, ws=24) == 1
    assert _attend(lib, _cache(B=0), q=0, out=0, ws=0, nbytes=0) == 0
    for shape in ((0, 8, 32, 8, 128, 100), (4, 0, 32, 8, 128, 100), (4, 8, 30, 8, 128, 100), (4, 257, 32, 8, 128, 100),
                  (4, 8, 32, 8, 96, 100), (4, 8, 32, 8, 128, 0), (4, 8, 32, 0, 128, 100)):
        assert lib.sd_tree_attention_workspace(*shape) == 0


def _accept(lib, z=16, dtype=0, B=2, R=5, V=100, stride=100, tokens=16, parents=16, n=0, emit=16, path=16, out=16, argmax=0,
            ws=16, nbytes=1 << 20):
    return lib.sd_accept_tree(P(z), dtype, B, R, V, stride, P(tokens), P(parents), P(n), P(emit), P(path), P(out), P(argmax),
                              P(ws), nbytes, None)


def test_accept(lib):
    assert _accept(lib, B=-1) == 1 and _accept(lib, R=0) == 1 and _accept(lib, V=0) == 1 and _accept(lib, stride=99) == 1
    assert _accept(lib, dtype=2) == 1 and _accept(lib, R=257) == 2 and _accept(lib, B=70000) == 2
    for name in ("z", "tokens", "emit", "path", "out"):
        assert _accept(lib, **{name: 0}) == 1
    assert _accept(lib, z=17) == 1 and _accept(lib, z=18, dtype=1) == 1
    assert _accept(lib, ws=0) == 3 and _accept(lib, nbytes=16) == 3 and _accept(lib, ws=24) == 3
    assert _accept(lib, B=0, z=0, ws=0) == 0
    assert lib.sd_accept_tree_workspace(3, 7, 100) >= 3 * 7 * 8 + 3 * 4
    assert lib.sd_accept_tree_workspace(0, 7, 100) == 0 and lib.sd_accept_tree_workspace(3, 0, 100) == 0


def test_commit(lib):
    def call(structs, path=16, emit=16, n=0, R=5, count=None):
        arr = (sd.PagedCacheStruct * max(len(structs), 1))(*structs)
        return lib.sd_paged_commit(arr, len(structs) if count is None else count, P(path), P(emit), P(n), R, None)
    one = lambda i, **kw: _struct(**{**dict(k=16 * i, v=1024 + 16 * i, n=4 * i, ticket=2048 + 4 * i), **kw})  # noqa: E731
    assert lib.sd_paged_commit(None, 1, P(16), P(16), None, 5, None) == 1
    assert call([], count=0) == 1 and call([one(1)], R=0) == 1 and call([one(1)], R=70000) == 2
    for kw, status in BAD_CACHES:
        assert call([one(1, **kw)]) == status, kw
    for kw in (dict(B=2), dict(H=4), dict(page=16), dict(D=64)):
        assert call([one(1), one(2, **kw)]) == 1                                # the caches disagree
    for kw in (dict(k=16), dict(v=1024 + 16), dict(n=4), dict(ticket=2048 + 4)):
        assert call([one(1), one(2, **kw)]) == 1, kw                            # one of them twice
    assert call([one(1)], path=0) == 1 and call([one(1)], emit=0) == 1
    assert call([one(1, B=0), one(2, B=0)], path=0, emit=0) == 0


def test_binding_refuses_what_it_can_see():
    k, t, n = torch.zeros(4, 1, 16, 64, dtype=torch.bfloat16), torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    for args in ((k, k[:3], t, n), (k[0], k[0], t, n), (k, k, t[0], n), (k, k, t, torch.zeros(2, dtype=torch.int32)), (k, k, t, n)):
        with pytest.raises(ValueError):
            sd.PagedKVCache(*args)  # (the last: on the CPU)
    with pytest.raises(ValueError):
        sd.PagedKVCache.empty(1, 1, 64, 64, page=0)
    with pytest.raises(ValueError):
        sd.PagedKVCacheGroup([])
    with pytest.raises(ValueError):
        sd.accept_tree(torch.zeros(1, 2, 8, dtype=torch.float16), torch.zeros(1, 2, dtype=torch.int32))
    with pytest.raises(ValueError):
        sd.accept_tree(torch.zeros(1, 2, 8), torch.zeros(1, 2, dtype=torch.int32))
