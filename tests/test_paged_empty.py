"""Appends of nothing: no rows or no scenes, with queries (whose address is then NULL)."""
import ctypes

import pytest
import torch

from paper_2606_31160_gb300 import build, sd

P = ctypes.c_void_p
SEC = (ctypes.c_int32 * 3)(16, 24, 24)


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return sd.lib()


def _append(lib, B=1, k=0, ks=1024, v=0, q=0, qs=4096, qo=0, R=0, Hq=32, pos=0, sec=SEC, inter=0):
    c = sd.PagedCacheStruct(16, 16, 16, 16, 16, B, 8, 40, 64, 4, 128)
    return lib.sd_paged_append(ctypes.byref(c), P(k), ks, P(v), 1024, P(q), qs, P(qo), R, Hq, P(pos), sec, inter, 1e6, None, None)


def test_nothing_to_append(lib):
    """The addresses of nothing may be NULL, queries' and positions' too; the rest is checked."""
    for nothing in (dict(R=0), dict(R=5, B=0), dict(R=0, B=0)):
        assert _append(lib, **nothing) == 0
        assert _append(lib, **nothing, qo=16) == 0 and _append(lib, **nothing, q=16, pos=16) == 0
        assert _append(lib, **nothing, Hq=0, qs=0) == 0
        assert _append(lib, **nothing, Hq=-1) == 1 and _append(lib, **nothing, inter=2) == 1
        assert _append(lib, **nothing, ks=1000) == 1
    assert _append(lib, R=-1) == 1


def test_what_goes_with_queries(lib):
    """With rows, as before: queries and their heads go together, and with positions."""
    rows = dict(R=5, k=16, v=16)
    assert _append(lib, **rows) == 1 and _append(lib, **rows, q=16, Hq=0, pos=16) == 1
    assert _append(lib, **rows, q=16) == 1 and _append(lib, **rows, Hq=0, qo=16) == 1
    assert _append(lib, **rows, q=16, pos=16, qs=4000) == 1 and _append(lib, **rows, q=16, pos=16, sec=None) == 1


@pytest.mark.gpu
@pytest.mark.parametrize("B,R", [(2, 0), (0, 3), (0, 0)])
@pytest.mark.parametrize("fused", [False, True])
def test_the_binding(B, R, fused):
    cache = sd.PagedKVCache(*(torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in "kv"),
                            torch.zeros((B, 2), dtype=torch.int32, device="cuda"), torch.full((B,), 3, dtype=torch.int32, device="cuda"))
    qkv = torch.zeros((B, R, 8, 64), dtype=torch.bfloat16, device="cuda")
    q, k, v = qkv.split([4, 2, 2], dim=2) if fused else (qkv[:, :, :4].contiguous(), qkv[:, :, 4:6].contiguous(), qkv[:, :, 6:].contiguous())
    pos = torch.zeros((B, R, 3), dtype=torch.int32, device="cuda")
    for q_out in (None, torch.empty((B, R, 4, 64), dtype=torch.bfloat16, device="cuda")):
        got = sd.paged_append(cache, k, v, q=q, pos=pos, sections=(8, 12, 12), q_out=q_out)
        assert got.shape == (B, R, 4, 64)
    assert sd.paged_append(cache, k, v) is None
    assert cache.len.tolist() == [3] * B and sd.get_device_error() == 0
