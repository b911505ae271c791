"""Host checks of the 8-bit cache, key weights, eviction and log probabilities: a bad
argument returns its status before anything is launched (no GPU needed), and the
binding refuses what it can see in the tensors."""
import ctypes

import pytest
import torch

from paper_2606_31160_gb300 import build, sd


@pytest.fixture(scope="module")
def lib():
    build.build()
    return sd.lib()


P = ctypes.c_void_p


def _c8(k=16, v=16, ks=16, vs=16, n=16, ticket=16, B=1, H=8, cap=200, D=128, block=64):
    return ctypes.byref(sd.KV8CacheStruct(k, v, ks, vs, n, ticket, B, H, cap, D, block))


def _c16(k=16, v=16, n=16, B=1, H=8, cap=200, D=128):
    return ctypes.byref(sd.KVCacheStruct(k, v, n, B, H, cap, D))


def test_kv8_append(lib):
    call = lambda c, k=16, v=16, R=8: lib.sd_kv8_append(c, P(k), P(v), R, None)  # noqa: E731
    assert call(None) == 1
    assert call(_c8(D=96)) == 2 and call(_c8(block=48)) == 2 and call(_c8(B=70000)) == 2
    assert call(_c8(cap=0)) == 1 and call(_c8(H=0)) == 1 and call(_c8(B=-1)) == 1
    assert call(_c8(), R=-1) == 1 and call(_c8(), R=201) == 1
    for field in ("k", "v", "ks", "vs", "n", "ticket"):
        assert call(_c8(**{field: 0})) == 1
    assert call(_c8(k=24)) == 1 and call(_c8(), k=0) == 1 and call(_c8(), v=8) == 1
    assert call(_c8(), R=0) == 0 and call(_c8(B=0, k=0)) == 0


def test_kv8_store(lib):
    call = lambda c, s: lib.sd_kv8_store(c, s, None)  # noqa: E731
    assert call(None, _c16()) == 1 and call(_c8(), None) == 1
    assert call(_c8(), _c16(B=2)) == 1 and call(_c8(), _c16(H=4)) == 1 and call(_c8(), _c16(D=64)) == 1
    assert call(_c8(), _c16(k=0)) == 1 and call(_c8(), _c16(v=8)) == 1 and call(_c8(), _c16(cap=0)) == 1
    assert call(_c8(B=0), _c16(B=0)) == 0


def test_kv8_attention(lib):
    def call(c, q=16, out=16, R=8, Hq=32, scale=0.0, flags=0):
        return lib.sd_kv8_attention(P(q), c, P(out), R, Hq, scale, flags, None)
    assert call(None) == 1 and call(_c8(D=32)) == 2 and call(_c8(block=16)) == 2
    assert call(_c8(), R=0) == 1 and call(_c8(), Hq=30) == 1 and call(_c8(), Hq=0) == 1
    assert call(_c8(), R=33) == 2                                    # G * R > 128
    assert call(_c8(), flags=2) == 1 and call(_c8(), flags=8) == 1
    assert call(_c8(), scale=-1.0) == 1 and call(_c8(), scale=float("nan")) == 1 and call(_c8(), scale=float("inf")) == 1
    assert call(_c8(), q=0) == 1 and call(_c8(), out=24) == 1
    assert call(_c8(B=0), q=0, out=0) == 0


def test_kv8_attention_with_a_workspace(lib):
    def call(c, q=16, out=16, R=8, Hq=32, scale=0.0, flags=0, ws=16, nbytes=1 << 24):
        return lib.sd_kv8_attention_ex(P(q), c, P(out), R, Hq, scale, flags, P(ws), nbytes, None)
    assert call(None) == 1 and call(_c8(D=32)) == 2 and call(_c8(), R=33) == 2
    assert call(_c8(), Hq=30) == 1 and call(_c8(), flags=2) == 1 and call(_c8(), scale=-1.0) == 1
    assert call(_c8(), q=0) == 1 and call(_c8(), ws=24) == 1
    assert call(_c8(B=0), q=0, out=0, ws=0, nbytes=0) == 0
    for shape in ((0, 8, 32, 8, 128, 100), (4, 0, 32, 8, 128, 100), (4, 8, 30, 8, 128, 100), (4, 33, 32, 8, 128, 100),
                  (4, 8, 32, 8, 96, 100), (4, 8, 32, 8, 128, 0), (4, 8, 32, 0, 128, 100)):
        assert lib.sd_kv8_attention_workspace(*shape) == 0


def test_attention_weights(lib):
    def call(c, q=16, R=8, Hq=32, scale=0.0, committed=0, before=16, decay=1.0, out=32):
        return lib.sd_attention_weights(P(q), c, R, Hq, scale, P(committed), P(before), decay, P(out), None)
    assert call(None) == 1 and call(_c16(D=96)) == 2 and call(_c16(B=70000)) == 2
    assert call(_c16(), R=0) == 1 and call(_c16(), Hq=30) == 1
    assert call(_c16(), scale=-1.0) == 1 and call(_c16(), decay=float("nan")) == 1
    assert call(_c16(), q=0) == 1 and call(_c16(k=0)) == 1 and call(_c16(n=0)) == 1 and call(_c16(), out=0) == 1
    assert call(_c16(), q=8) == 1 and call(_c16(k=8)) == 1
    assert call(_c16(B=0), q=0, out=0) == 0


def test_attention_weights_with_a_workspace(lib):
    def call(c, q=16, R=8, Hq=32, out=32, ws=16, nbytes=1 << 20):
        return lib.sd_attention_weights_ex(P(q), c, R, Hq, 0.0, P(0), P(0), 1.0, P(out), P(ws), nbytes, None)
    assert call(None) == 1 and call(_c16(D=96)) == 2 and call(_c16(), R=0) == 1 and call(_c16(), Hq=30) == 1
    assert call(_c16(), q=0) == 1 and call(_c16(), out=0) == 1 and call(_c16(), ws=24) == 1
    assert call(_c16(B=0), q=0, out=0, ws=0, nbytes=0) == 0
    for shape in ((0, 8, 32, 8, 128, 100), (4, 0, 32, 8, 128, 100), (4, 8, 30, 8, 128, 100), (4, 33, 32, 8, 128, 100),
                  (4, 8, 32, 8, 96, 100), (4, 8, 32, 8, 128, 0), (4, 8, 32, 0, 128, 100)):
        assert lib.sd_attention_weights_workspace(*shape) == 0


def test_kv_evict(lib):
    big = 1 << 30
    src = dict(k=big, v=2 * big, n=16)
    dst = dict(k=3 * big, v=4 * big, n=32, cap=100)

    def call(s=src, d=dst, w=5 * big, keep=50, sinks=4, recent=8, wo=6 * big, kept=7 * big, **more):
        return lib.sd_kv_evict(_c16(**{**s, **more}), P(w), keep, sinks, recent, _c16(**d), P(wo), P(kept), None)
    assert lib.sd_kv_evict(None, P(16), 5, 0, 0, _c16(**dst), None, None, None) == 1
    assert lib.sd_kv_evict(_c16(**src), P(16), 5, 0, 0, None, None, None, None) == 1
    assert call(B=2) == 1 and call(H=4) == 1 and call(D=64) == 1      # the caches disagree
    assert call(d={**dst, "D": 96}, D=96) == 2
    assert call(keep=0) == 1 and call(keep=101) == 1 and call(sinks=-1) == 1 and call(recent=-1) == 1
    assert call(sinks=43, recent=8) == 1                             # more protected than kept
    assert call(w=0) == 1 and call(k=0) == 1 and call(d={**dst, "v": 0}) == 1 and call(d={**dst, "k": 3 * big + 8}) == 1
    assert call(d={**dst, "k": big + 4096}) == 1                     # writes what it reads
    assert call(wo=5 * big + 64) == 1 and call(kept=2 * big) == 1 and call(d={**dst, "n": 16}) == 1
    assert call(d={**dst, "B": 0}, B=0) == 0


def test_token_logprobs(lib):
    def call(z=16, dtype=0, rows=3, V=100, stride=100, tokens=16, T=1.0, n=4, lp=16, h=16, ids=16, tops=16):
        return lib.sd_token_logprobs(P(z), dtype, rows, V, stride, P(tokens), T, n, P(lp), P(h), P(ids), P(tops), None)
    assert call(rows=-1) == 1 and call(V=0) == 1 and call(stride=99) == 1 and call(dtype=2) == 1
    for T in (0.0, -1.0, float("nan"), float("inf"), 1e-45):
        assert call(T=T) == 1
    assert call(n=-1) == 1 and call(n=33) == 2 and call(V=3, n=4) == 1
    assert call(z=0) == 1 and call(tokens=0) == 1 and call(lp=0) == 1 and call(ids=0) == 1 and call(tops=0) == 1
    assert call(rows=0, z=0) == 0


def test_binding_refuses_cpu_tensors_and_shapes():
    z = torch.zeros(2, 3, 10)
    with pytest.raises(ValueError):
        sd.token_logprobs(z, torch.zeros(2, 3, dtype=torch.int32))
    with pytest.raises(ValueError):
        sd.token_logprobs(z.double(), torch.zeros(2, 3, dtype=torch.int32))
    with pytest.raises(ValueError):
        sd.token_logprobs(z, torch.zeros(2, 4, dtype=torch.int32))
    with pytest.raises(ValueError):
        sd.KV8Cache.empty(1, 1, 64, 128, device="cpu")
    k = torch.zeros(1, 1, 64, 128, dtype=torch.uint8).view(torch.float8_e4m3fn)
    with pytest.raises(ValueError):
        sd.KV8Cache(k, k, torch.ones(1, 1, 2), torch.ones(1, 1, 2), torch.zeros(1, dtype=torch.int32), block=64)
