"""GPU parity of the accumulated key weights and the eviction against the float64 oracle."""
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


# ------------------------------------------------------------------ weights

@pytest.mark.parametrize("D,cap,R,Hq,Hkv,lens", [
    (128, 300, 1, 4, 1, [1, 2, 127, 128, 129, 300]),
    (128, 4113, 8, 32, 8, [4104, 8]),
    (64, 1200, 6, 28, 4, [6, 1200, 129]),
    (128, 700, 33, 8, 8, [700, 33, 64]),
    (64, 515, 70, 3, 1, [515, 70]),
    (128, 9000, 3, 2, 2, [9000, 8191]),
    (128, 20011, 2, 4, 1, [20011, 16384]),
])
@pytest.mark.parametrize("spread", [1.0, 20.0])
def test_weights_parity(D, cap, R, Hq, Hkv, lens, spread):
    rng = np.random.default_rng(cap + R)
    B = len(lens)
    k = _bf16(rng.standard_normal((B, Hkv, cap, D)))
    for b, n in enumerate(lens):
        k[b, :, n:] = float("nan")
    q = _bf16(rng.standard_normal((B, R, Hq, D)) * spread)
    cache = sd.KVCache(k, k.clone(), _i32(lens))
    before = torch.from_numpy(rng.random((B, Hkv, cap)).astype(np.float32)).cuda()
    for b, n in enumerate(lens):
        before[b, :, n - R:] = float("nan")  # rolled back: never read
    committed = [int(rng.integers(0, R + 1)) for _ in lens]
    k64 = np.nan_to_num(to64(k))
    for com, bef, decay in ((None, None, 1.0), (committed, before, 0.75)):
        out = torch.full((B, Hkv, cap), -5.0, device="cuda")
        sd.attention_weights(q, cache, bef, out, decay, None if com is None else _i32(com))
        ref = oracle.attention_weights(to64(q), k64, lens, com, None if bef is None else to64(bef), decay)
        got = to64(out)
        rows = R * Hq // Hkv
        for b, n in enumerate(lens):
            assert (got[b, :, n:] == -5.0).all()
            # fp32 scores: an error of a few 2^-23 of sum |q k| scale, which is an error
            # of as many parts in one of a weight; then sums of `rows` weights
            big = 2.0 ** -21 * np.abs(to64(q[b])).max() * np.abs(k64[b]).max() * D / np.sqrt(D)
            tol = (1e-5 + min(big, 1e-3)) * ref[b, :, :n] + 1e-7 * rows
            assert np.all(np.abs(got[b, :, :n] - ref[b, :, :n]) <= tol)
    assert sd.get_device_error() == 0


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("size", [1, 2])
@pytest.mark.parametrize("Hq,R", [(6, 50), (2, 32), (4, 8)])
def test_weights_tiles_kept_between_readings(D, size, Hq, R):
    """One to eleven tiles of keys a CTA, one to three groups of rows: keys that stay in
    shared memory between the readings, and those that are read again."""
    rng = np.random.default_rng(D + R)
    lens = [60, 128, 300, 400, 513, 640, 700, 896, 1000, 1150, 1280, 1400]
    k = _bf16(rng.standard_normal((len(lens), 1, 1400, D)))
    q = _bf16(rng.standard_normal((len(lens), R, Hq, D)))
    sd.set_cluster_size(size)
    try:
        got = to64(sd.attention_weights(q, sd.KVCache(k, k.clone(), _i32(lens))))
    finally:
        sd.set_cluster_size(0)
    assert sd.get_device_error() == 0
    ref = oracle.attention_weights(to64(q), to64(k), lens)
    for b, n in enumerate(lens):
        big = 2.0 ** -21 * np.abs(to64(q[b])).max() * np.abs(to64(k[b])).max() * np.sqrt(D)
        tol = (1e-5 + min(big, 1e-3)) * ref[b, :, :n] + 1e-7 * R * Hq
        assert np.all(np.abs(got[b, :, :n] - ref[b, :, :n]) <= tol)


def test_weights_in_place_and_accumulating():
    rng = np.random.default_rng(3)
    k = _bf16(rng.standard_normal((2, 2, 400, 128)))
    q = _bf16(rng.standard_normal((2, 4, 8, 128)))
    cache = sd.KVCache(k, k.clone(), _i32([400, 300]))
    once = sd.attention_weights(q, cache)
    acc = once.clone()
    sd.attention_weights(q, cache, weights_in=acc, weights=acc, decay=1.0)
    for b, n in ((0, 400), (1, 300)):
        assert torch.allclose(acc[b, :, :n - 4], 2 * once[b, :, :n - 4], rtol=1e-6, atol=0)
        assert torch.equal(acc[b, :, n - 4:n], once[b, :, n - 4:n])
        assert torch.allclose(once[b, :, :n].sum(-1), torch.full((2,), 16.0, device="cuda"), rtol=1e-4)
        assert (once[b, :, n:] == 0).all()


def test_weights_bad_scenes():
    rng = np.random.default_rng(4)
    k = _bf16(rng.standard_normal((4, 1, 100, 64)))
    q = _bf16(rng.standard_normal((4, 5, 2, 64)))
    out = torch.full((4, 1, 100), 7.0, device="cuda")
    sd.attention_weights(q, sd.KVCache(k, k.clone(), _i32([4, 101, 60, 60])), weights=out, committed=_i32([5, 5, 6, 5]))
    assert sd.get_device_error() == sd.SD_DEVERR_LENGTH | sd.SD_DEVERR_ROLLBACK
    assert (out[:3] == 7.0).all() and (out[3, 0, :60] != 7.0).all()


def test_weights_are_deterministic():
    rng = np.random.default_rng(5)
    k = _bf16(rng.standard_normal((3, 4, 5000, 128)))
    q = _bf16(rng.standard_normal((3, 9, 16, 128)))
    cache = sd.KVCache(k, k.clone(), _i32([5000, 3000, 777]))
    first = sd.attention_weights(q, cache)
    for _ in range(3):
        assert torch.equal(sd.attention_weights(q, cache), first)


# ------------------------------------------------------------------ eviction

def _evict(w, lens, keep, sinks, recent, D=64, cap2=None, extra=True):
    B, H, cap = w.shape
    rng = np.random.default_rng(cap)
    k, v = _bf16(rng.standard_normal((B, H, cap, D))), _bf16(rng.standard_normal((B, H, cap, D)))
    cap2 = keep + 3 if cap2 is None else cap2
    dst = sd.KVCache(torch.full((B, H, cap2, D), 9.0, dtype=torch.bfloat16, device="cuda"),
                     torch.full((B, H, cap2, D), 9.0, dtype=torch.bfloat16, device="cuda"), _i32([-1] * B))
    wt = torch.from_numpy(w.astype(np.float32)).cuda()
    w2 = torch.full((B, H, cap2), -3.0, device="cuda") if extra else None
    kept = torch.full((B, H, keep), -9, dtype=torch.int32, device="cuda") if extra else None
    sd.kv_evict(sd.KVCache(k, v, _i32(lens)), wt, dst, keep, sinks, recent, w2, kept)
    for b, n in enumerate(lens):
        m = min(n, keep)
        assert dst.len[b].item() == m
        for h in range(H):
            want = oracle.kept_keys(w[b, h], n, keep, sinks, recent)
            at = torch.from_numpy(want).cuda()
            if extra:
                assert kept[b, h].tolist() == want.tolist() + [-1] * (keep - m)
                assert torch.equal(w2[b, h, :m].nan_to_num(nan=-7.0), wt[b, h, at].nan_to_num(nan=-7.0)) and (w2[b, h, m:] == -3.0).all()
            assert torch.equal(dst.k[b, h, :m], k[b, h, at]) and torch.equal(dst.v[b, h, :m], v[b, h, at])
            assert (dst.k[b, h, m:] == 9.0).all() and (dst.v[b, h, m:] == 9.0).all()
    assert sd.get_device_error() == 0


@pytest.mark.parametrize("cap,lens,keep,sinks,recent,D", [
    (300, [300, 1, 0, 40, 41, 299], 40, 4, 8, 64),
    (4200, [4113, 2048, 2049], 2048, 4, 64, 128),
    (1025, [1025, 1024, 1023], 1, 0, 0, 64),
    (700, [700, 650], 700, 0, 0, 128),
    (100, [100, 64], 64, 64, 0, 64),
    (100, [100, 64, 65], 64, 0, 64, 64),
    (20011, [20011, 16385], 5003, 7, 1000, 64),
])
@pytest.mark.parametrize("kind", ["random", "ties", "equal"])
def test_evict_parity(cap, lens, keep, sinks, recent, D, kind):
    rng = np.random.default_rng(cap + keep)
    w = {"random": np.exp(2 * rng.standard_normal((len(lens), 2, cap))),
         "ties": rng.integers(0, 4, (len(lens), 2, cap)) * 0.25,
         "equal": np.ones((len(lens), 2, cap))}[kind]
    _evict(w, lens, keep, sinks, recent, D)


def test_evict_special_weights():
    rng = np.random.default_rng(9)
    w = rng.standard_normal((2, 3, 257))  # negative ones order too
    w[:, :, 5:50:5] = np.nan
    w[:, :, 7] = np.inf
    w[:, :, 9:80:7] = -np.inf
    w[:, :, 100:140] = 0.0
    w[:, :, 101:140:3] = -0.0
    for keep in (1, 60, 150, 200, 230, 250):
        _evict(w, [257, 130], keep, 0, 0)


@pytest.mark.parametrize("cap", [127, 128, 129, 515, 5000, 21000])
@pytest.mark.parametrize("kind", ["crowded", "far", "nan", "low", "negative"])
def test_evict_ranges_of_weights(cap, kind):
    """The selection counts weights by equal ranges between the least and the largest."""
    rng = np.random.default_rng(cap)
    if kind == "crowded":    # all but two in one range, few of them alike
        w = (1.0 + rng.integers(0, 4000, (1, 2, cap)) * 2.0 ** -23).astype(np.float32)
        w[:, :, 1], w[:, :, 2] = 1e30, 1e-30
    elif kind == "far":      # infinities, denormals, zeros of both signs
        w = np.exp(rng.standard_normal((1, 2, cap)) * 30).astype(np.float32)
        w[:, :, ::5], w[:, :, 1::7], w[:, :, 2::11], w[:, 0, 3], w[:, 1, 4] = 0.0, -0.0, 1e-42, np.inf, -np.inf
    elif kind == "nan":      # more keys are kept than have a number
        w = np.full((1, 2, cap), np.nan, dtype=np.float32)
        w[:, :, ::9] = rng.random(w[:, :, ::9].shape)
    elif kind == "low":      # every weight -inf but one
        w = np.full((1, 2, cap), -np.inf, dtype=np.float32)
        w[:, :, cap // 2] = -1e38
    else:
        w = -rng.random((1, 2, cap)).astype(np.float32)
    for keep, sinks, recent in ((1, 0, 0), (cap // 2, 3, 5), (cap - 1, 0, 0), (cap - 1, cap // 3, cap // 3)):
        _evict(w, [cap], keep, sinks, recent)


def test_evict_without_extras_and_into_a_smaller_capacity():
    rng = np.random.default_rng(10)
    _evict(rng.random((2, 2, 500)), [500, 77], 100, 2, 3, cap2=100, extra=False)


def test_evict_bad_lengths():
    k = torch.zeros((3, 1, 50, 64), dtype=torch.bfloat16, device="cuda")
    dst = sd.KVCache(torch.zeros((3, 1, 9, 64), dtype=torch.bfloat16, device="cuda"),
                     torch.zeros((3, 1, 9, 64), dtype=torch.bfloat16, device="cuda"), _i32([5, 5, 5]))
    sd.kv_evict(sd.KVCache(k, k.clone(), _i32([51, -1, 50])), torch.rand((3, 1, 50), device="cuda"), dst, 9)
    assert sd.get_device_error() == sd.SD_DEVERR_LENGTH and dst.len.tolist() == [5, 5, 9]


def test_attention_over_the_kept_keys():
    """weights -> evict -> 8-bit store -> attention: what stays answers nearly as the whole
    did where the evicted keys had little weight."""
    rng = np.random.default_rng(12)
    B, H, L, D, R = 2, 2, 1000, 128, 4
    k = rng.standard_normal((B, H, L, D))
    k[:, :, 300:] *= 0.01  # near-constant small scores
    q = rng.standard_normal((B, R, 4, D))
    q[..., :] += 0.0
    k[:, :, ::10] += 3 * q[:, :1, ::2].transpose(0, 2, 1, 3)  # heavy keys
    cache = sd.KVCache(_bf16(k), _bf16(rng.standard_normal((B, H, L, D))), _i32([L, L - 100]))
    qd = _bf16(q)
    w = sd.attention_weights(qd, cache)
    dst = sd.KVCache.empty(B, H, 500, D)
    sd.kv_evict(cache, w, dst, 400, sinks=4, recent=R)
    c8 = sd.KV8Cache.empty(B, H, 420, D)
    sd.kv8_store(c8, dst)
    small = sd.kv8_attention(qd, c8)
    codes = lambda t, s: oracle.dequantise(t.float().cpu().numpy().astype(np.float64), s.cpu().numpy().astype(np.float64), 64)  # noqa: E731
    ref = oracle.verify_attention(to64(qd), codes(c8.k, c8.k_scale), codes(c8.v, c8.v_scale), c8.len.cpu().numpy())
    assert np.abs(to64(small) - ref).max() <= 3e-2
    assert c8.len.tolist() == [400, 400] and sd.get_device_error() == 0
