"""The 8-bit cache, key weights, eviction and log probabilities where indexes pass 32
bits, at every cluster size, on other streams and in graphs, and with numbers that are
none."""
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


def _bf16(x):
    return workloads.to_bf16(np.asarray(x, dtype=np.float32)).cuda()


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _codes(t):
    return t.float().cpu().numpy().astype(np.float64)


def _cache8(rng, B, H, cap, D, block, lens):
    c = sd.KV8Cache.empty(B, H, cap, D, block)
    for t in (c.k, c.v):
        x = oracle.round_e4m3(np.clip(rng.standard_normal((B, H, cap, D)) * 100, -448, 448))
        t.copy_(torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).cuda())
    c.k_scale.fill_(2.0 ** -7)
    c.v_scale.fill_(2.0 ** -7)
    c.len.copy_(_i32(lens))
    return c


def _attention_close(out, q, k, v, lens, **kw):
    ref = oracle.verify_attention(to64(q), k, v, lens, **kw)
    mag = oracle.verify_attention(to64(q), k, np.abs(v), lens, **kw)
    # the output's rounding, one of 2^-8 a weight, and weights of subnormal terms: 2^-13 of the
    # largest value and key, added as random errors
    tol = 2.0 ** -8 * np.abs(ref) + 2.0 ** -8 * mag + 2.0 ** -13 * np.sqrt(max(lens)) * np.abs(v).max()
    assert np.all(np.abs(to64(out) - ref) <= tol)


def test_offsets_past_32_bits_in_the_8_bit_cache():
    """The last head's rows lie past 2^31 bytes from the first's."""
    rng = np.random.default_rng(0)
    H, cap, D, n, R = 9, 2_000_003, 128, 700, 5
    k = torch.empty((1, H, cap, D), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    v = torch.empty_like(k)
    s = torch.empty((1, H, -(-cap // 64)), device="cuda")
    c = sd.KV8Cache(k, v, s, torch.empty_like(s), torch.zeros(1, dtype=torch.int32, device="cuda"))
    prefix = [_bf16(rng.standard_normal((1, n, H, D))) for _ in range(2)]
    new = [_bf16(rng.standard_normal((1, R, H, D))) for _ in range(2)]
    sd.kv8_append(c, *prefix)
    sd.kv8_append(c, *new)
    q = _bf16(rng.standard_normal((1, R, 4 * H, D)))
    out = sd.kv8_attention(q, c)
    vals = []
    for t, sc, p, x in ((c.k, c.k_scale, prefix[0], new[0]), (c.v, c.v_scale, prefix[1], new[1])):
        codes, scales = np.zeros((1, H, n + R, D)), np.ones((1, H, -(-(n + R) // 64)))
        codes, scales = oracle.kv8_append(codes, scales, [0], to64(p), 64)
        codes, scales = oracle.kv8_append(codes, scales, [n], to64(x), 64)
        assert np.array_equal(_codes(t[:, :, :n + R]), codes)
        vals.append(oracle.dequantise(codes, scales, 64))
    _attention_close(out, q, *vals, [n + R])
    # rows far into one head, past 2^31 bytes of it too, and their neighbours
    c.len.fill_(cap - R)
    c.k_scale.fill_(1.0)
    c.v_scale.fill_(1.0)
    sd.kv8_append(c, *new)
    assert c.len.item() == cap
    want, _ = oracle.kv8_append(np.zeros((1, H, 128, D)), np.ones((1, H, 2)), [(cap - R) % 64], to64(new[0]), 64)
    assert np.array_equal(_codes(c.k[:, :, cap - R:]), want[:, :, (cap - R) % 64:(cap - R) % 64 + R])
    assert sd.get_device_error() == 0


def test_offsets_past_32_bits_in_eviction_and_weights():
    rng = np.random.default_rng(1)
    H, cap, D, n, keep, R = 17, 1_100_001, 128, 900, 300, 4
    k = torch.empty((1, H, cap, D), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    k[:, :, :n] = _bf16(rng.standard_normal((1, H, n, D)))
    v[:, :, :n] = _bf16(rng.standard_normal((1, H, n, D)))
    cache = sd.KVCache(k, v, _i32([n]))
    q = _bf16(rng.standard_normal((1, R, 2 * H, D)))
    w = sd.attention_weights(q, cache, weights=torch.empty((1, H, cap), device="cuda"))
    ref = oracle.attention_weights(to64(q), to64(k[:, :, :n]), [n])
    got = w[:, :, :n].cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got - ref) <= 2e-5 * ref + 1e-6)
    dst = sd.KVCache(torch.empty_like(k), torch.empty_like(v), _i32([0]))
    kept = torch.empty((1, H, keep), dtype=torch.int32, device="cuda")
    sd.kv_evict(cache, w, dst, keep, kept=kept)
    for h in (0, 8, H - 1):
        want = oracle.kept_keys(got[0, h], n, keep, 0, 0)
        at = torch.from_numpy(want).cuda()
        assert kept[0, h].tolist() == want.tolist()
        assert torch.equal(dst.k[0, h, :keep], k[0, h, at]) and torch.equal(dst.v[0, h, :keep], v[0, h, at])
    assert sd.get_device_error() == 0


def test_evicting_most_of_a_long_cache():
    """More keys than stay in shared memory, and lists of more than one round."""
    rng = np.random.default_rng(2)
    n, keep = 70_001, 9_000
    w = rng.random(n).astype(np.float32)
    w[::7] = 0.5
    k = _bf16(rng.standard_normal((1, 1, n, 64)))
    dst = sd.KVCache.empty(1, 1, keep, 64)
    kept = torch.empty((1, 1, keep), dtype=torch.int32, device="cuda")
    for weights in (w, np.round(w, 2), np.ones(n, dtype=np.float32)):
        sd.kv_evict(sd.KVCache(k, k.clone(), _i32([n])), torch.from_numpy(weights).cuda().view(1, 1, n), dst, keep, 3, 5, kept=kept)
        want = oracle.kept_keys(weights.astype(np.float64), n, keep, 3, 5)
        assert np.array_equal(kept.cpu().numpy()[0, 0], want)
        assert torch.equal(dst.k[0, 0], k[0, 0, torch.from_numpy(want).cuda()])


@pytest.mark.parametrize("cs", [1, 2, 4, 6, 8, 16])
def test_every_cluster_size(cs):
    rng = np.random.default_rng(3)
    sd.set_cluster_size(cs)
    try:
        for D, Hq, Hkv, R, lens in ((128, 8, 2, 8, [3001, 40, 9]), (64, 12, 2, 7, [2500, 7, 1111]), (128, 7, 1, 17, [1700, 300])):
            c = _cache8(rng, len(lens), Hkv, max(lens), D, 64, lens)
            q = _bf16(rng.standard_normal((len(lens), R, Hq, D)))
            out = sd.kv8_attention(q, c)
            k, v = (oracle.dequantise(_codes(t), np.full(c.k_scale.shape, 2.0 ** -7), 64) for t in (c.k, c.v))
            _attention_close(out, q, k, v, lens)
            kb = _bf16(rng.standard_normal((len(lens), Hkv, max(lens), D)))
            w = sd.attention_weights(q, sd.KVCache(kb, kb.clone(), _i32(lens)))
            ref = oracle.attention_weights(to64(q), to64(kb), lens)
            for b, n in enumerate(lens):
                assert np.all(np.abs(to64(w)[b, :, :n] - ref[b, :, :n]) <= 2e-5 * ref[b, :, :n] + 1e-6 * R)
    finally:
        sd.set_cluster_size(0)
    assert sd.get_device_error() == 0


def test_other_streams_and_graphs():
    """Each operator on a side stream, and captured once and replayed, gives what it gave."""
    rng = np.random.default_rng(4)
    B, Hq, Hkv, D, L, R, V = 2, 8, 2, 128, 900, 4, 7001
    kb, vb = (_bf16(rng.standard_normal((B, Hkv, L, D))) for _ in range(2))
    cache = sd.KVCache(kb, vb, _i32([L, L - 77]))
    q = _bf16(rng.standard_normal((B, R, Hq, D)))
    z, tok = _bf16(rng.standard_normal((B, R, V))), torch.randint(0, V, (B, R), device="cuda").to(torch.int32)
    dst, c8 = sd.KVCache.empty(B, Hkv, 300, D), sd.KV8Cache.empty(B, Hkv, 300, D)
    w = torch.zeros((B, Hkv, L), device="cuda")
    out = torch.empty_like(q)
    lp = [torch.empty((B, R), device="cuda"), torch.empty((B, R), device="cuda"),
          torch.empty((B, R, 6), dtype=torch.int32, device="cuda"), torch.empty((B, R, 6), device="cuda")]

    def chain():
        sd.attention_weights(q, cache, weights=w)
        sd.kv_evict(cache, w, dst, 300, recent=R)
        sd.kv8_store(c8, dst)
        sd.kv8_attention(q, c8, out=out)
        sd.token_logprobs(z, tok, 0.8, 6, *lp)

    def state():
        return [t.clone() for t in (w, dst.k, c8.k.view(torch.uint8), c8.k_scale, out, *lp)]
    chain()
    want = state()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out.zero_()
        chain()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(state(), want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        chain()
    for t in (w, dst.k, out, *lp):
        t.zero_()
    for _ in range(3):
        g.replay()
    assert all(torch.equal(a, b) for a, b in zip(state(), want))
    assert sd.get_device_error() == 0


def test_numbers_that_are_none_stay_where_they_are():
    rng = np.random.default_rng(5)
    c = _cache8(rng, 1, 2, 500, 128, 64, [500])
    q = _bf16(rng.standard_normal((1, 6, 8, 128)))
    good = sd.kv8_attention(q, c).clone()
    bad = q.clone()
    bad[0, 2, 1, 5] = float("nan")
    bad[0, 3, 6, 7] = float("inf")
    out = sd.kv8_attention(bad, c)
    assert out[0, 2, 1].isnan().all() and out[0, 3, 6].isnan().all()
    rows = torch.ones((6, 8), dtype=torch.bool, device="cuda")
    rows[2, 1] = rows[3, 6] = False
    # (a tile with such a row scales its rows one by one: the same numbers to fp32 rounding)
    assert torch.allclose(out[0][rows].float(), good[0][rows].float(), rtol=2.0 ** -7, atol=2.0 ** -10)
    c.v.view(torch.uint8)[0, 0, 77, 3] = 0x7f          # one value: its column, in the head's rows
    out = sd.kv8_attention(q, c)
    assert out[0, :, :4, 3].isnan().all() and torch.equal(out[0, :, 4:], good[0, :, 4:])
    assert torch.equal(out[0, :, :4, :3], good[0, :, :4, :3]) and torch.equal(out[0, :, :4, 4:], good[0, :, :4, 4:])
    c.k.view(torch.uint8)[0, 1, 497, 3] = 0xff         # one key: the rows that see it
    out = sd.kv8_attention(q, c)
    assert out[0, 3:, 4:].isnan().all() and torch.equal(out[0, :3, 4:], good[0, :3, 4:])
    # key weights: a key that is no number takes the rows that see it with it
    k = _bf16(rng.standard_normal((1, 1, 300, 128)))
    k[0, 0, 298, 9] = float("nan")
    qw = _bf16(rng.standard_normal((1, 4, 2, 128)))
    cache = sd.KVCache(k, k.clone(), _i32([300]))
    assert sd.attention_weights(qw, cache).isnan().all()
    seen = sd.attention_weights(qw, cache, committed=_i32([2]))[0, 0]
    assert not seen[:298].isnan().any() and (seen[298:] == 0).all()
    assert sd.get_device_error() == 0


def test_empty_and_single():
    """Lengths of 0 and 1; one row, one key, one token."""
    rng = np.random.default_rng(6)
    k = _bf16(rng.standard_normal((2, 1, 4, 64)))
    cache = sd.KVCache(k, k.clone(), _i32([0, 1]))
    dst, c8 = sd.KVCache.empty(2, 1, 3, 64), sd.KV8Cache.empty(2, 1, 4, 64, block=32)
    kept = torch.empty((2, 1, 3), dtype=torch.int32, device="cuda")
    sd.kv_evict(cache, torch.rand((2, 1, 4), device="cuda"), dst, 3, kept=kept)
    assert dst.len.tolist() == [0, 1] and kept.tolist() == [[[-1, -1, -1]], [[0, -1, -1]]]
    sd.kv8_store(c8, cache)
    assert c8.len.tolist() == [0, 1]
    sd.kv8_append(c8, _bf16(np.ones((2, 1, 1, 64))), _bf16(np.full((2, 1, 1, 64), 3.0)))
    out = sd.kv8_attention(_bf16(rng.standard_normal((2, 1, 3, 64))), c8)
    assert (out[0] == 3.0).all() and c8.len.tolist() == [1, 2]  # one key: its value
    w = sd.attention_weights(_bf16(rng.standard_normal((1, 1, 3, 64))), sd.KVCache(k[:1], k[:1].clone(), _i32([1])))
    assert torch.allclose(w[0, 0], torch.tensor([3.0, 0, 0, 0], device="cuda"))
    lp, h, ids, top = sd.token_logprobs(torch.full((1, 1), 5.0, device="cuda"), _i32([0]), top_n=1)
    assert lp.item() == 0 and h.item() == 0 and ids.item() == 0 and top.item() == 0
    assert sd.get_device_error() == 0
