"""GPU parity of the 8-bit KV cache: append, store and the attention over it, against the
float64 oracle."""
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


def _codes(t):
    return t.float().cpu().numpy().astype(np.float64)


def _cache(rng, B, H, cap, D, block, spread=1.0, lens=None):
    """A cache whose every row is valid, random codes under random power-of-two scales."""
    c = sd.KV8Cache.empty(B, H, cap, D, block)
    x = oracle.round_e4m3(np.clip(rng.standard_normal((B, H, cap, D)) * 100, -448, 448))
    for t in (c.k, c.v):
        t.copy_(torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).cuda())
        x = x[..., ::-1].copy()
    c.k_scale.copy_(torch.from_numpy((2.0 ** rng.integers(-8, -5, c.k_scale.shape) * spread).astype(np.float32)))
    c.v_scale.copy_(torch.from_numpy((2.0 ** rng.integers(-9, -5, c.k_scale.shape)).astype(np.float32)))
    if lens is not None:
        c.len.copy_(torch.tensor(lens, dtype=torch.int32))
    return c


# one row; a row that ends and one that begins a block; rows over several blocks; a last
# block cut off by the capacity; scenes at every offset within a block
@pytest.mark.parametrize("D,block,cap,R,lens", [
    (128, 64, 200, 8, [0, 1, 57, 63, 64, 120, 192]),
    (64, 32, 133, 1, [0, 31, 32, 33, 132]),
    (64, 64, 300, 150, [0, 10, 150, 63]),
    (128, 128, 257, 129, [0, 127, 128, 100]),
    (128, 32, 70, 70, [0]),
    (64, 128, 90, 17, [5, 73]),
])
@pytest.mark.parametrize("mag", [1.0, 1e-3, 300.0])
def test_append_bit_exact(D, block, cap, R, lens, mag):
    rng = np.random.default_rng(R * 7 + block)
    B, H = len(lens), 3
    c = _cache(rng, B, H, cap, D, block, lens=lens)
    k_new, v_new = _bf16(rng.standard_normal((B, R, H, D)) * mag), _bf16(rng.standard_normal((B, R, H, D)) * mag * 0.1)
    want = [oracle.kv8_append(_codes(t), s.cpu().numpy(), lens, to64(n), block)
            for t, s, n in ((c.k, c.k_scale, k_new), (c.v, c.v_scale, v_new))]
    sd.kv8_append(c, k_new, v_new)
    for (codes, scales), t, s in ((want[0], c.k, c.k_scale), (want[1], c.v, c.v_scale)):
        assert np.array_equal(s.cpu().numpy(), scales.astype(np.float32))
        assert np.array_equal(_codes(t), codes)
    assert c.len.tolist() == [n + R for n in lens] and not c._ticket.any() and sd.get_device_error() == 0


def test_append_special_values_and_growth_from_zeros():
    rng = np.random.default_rng(5)
    c = sd.KV8Cache.empty(1, 1, 64, 64, 64)
    steps = [np.zeros((1, 2, 1, 64)), rng.standard_normal((1, 3, 1, 64)) * 1e-30, rng.standard_normal((1, 2, 1, 64)),
             rng.standard_normal((1, 1, 1, 64)) * 3e38]
    steps[2][0, 0, 0, :4] = [np.inf, -np.inf, np.nan, 0.0]
    codes, scales, n = np.zeros((1, 1, 64, 64)), np.ones((1, 1, 1)), 0
    for x in steps:
        new = _bf16(x)
        codes, scales = oracle.kv8_append(codes, scales, [n], to64(new), 64)
        sd.kv8_append(c, new, new)
        n += x.shape[1]
        assert np.array_equal(_codes(c.k), codes, equal_nan=True) and np.array_equal(_codes(c.v), codes, equal_nan=True)
        assert c.k_scale.item() == scales[0, 0, 0]
    assert sd.get_device_error() == 0


def test_append_under_a_scale_that_is_no_power_of_two():
    rng = np.random.default_rng(6)
    for s0, mag in ((0.3, 1.0), (0.013, 500.0)):
        c = _cache(rng, 1, 2, 128, 128, 64, lens=[70])
        c.k_scale.fill_(s0)
        new = _bf16(rng.standard_normal((1, 5, 2, 128)) * mag)
        a = new.float().abs().amax((1, 3))[0].cpu().numpy().astype(np.float64)
        s = np.float32(s0)
        g = [max(0, int(np.ceil(np.log2(x / 448 / np.float64(s))))) for x in a]
        sd.kv8_append(c, new, new)
        for h in range(2):
            want = np.float32(s * np.float32(2.0 ** g[h]))
            assert c.k_scale[0, h, 1].item() == want
            q = (new[0, :, h].float().cpu().numpy() / want).astype(np.float32)  # fp32's division, then one rounding
            assert np.array_equal(_codes(c.k)[0, h, 70:75], oracle.round_e4m3(q))


def test_append_overflow_leaves_the_scene():
    rng = np.random.default_rng(7)
    c = _cache(rng, 3, 2, 100, 64, 32, lens=[90, 93, 40])
    before, scales = c.k.view(torch.uint8).clone(), c.k_scale.clone()
    new = _bf16(rng.standard_normal((3, 8, 2, 64)))
    sd.kv8_append(c, new, new)
    assert sd.get_device_error() == sd.SD_DEVERR_KV_OVERFLOW
    assert c.len.tolist() == [98, 93, 48] and not c._ticket.any()
    assert torch.equal(c.k.view(torch.uint8)[1], before[1]) and torch.equal(c.k_scale[1], scales[1])
    for b, n in ((0, 90), (2, 40)):
        assert torch.equal(c.k.view(torch.uint8)[b, :, n + 8:], before[b, :, n + 8:])
        assert torch.equal(c.k.view(torch.uint8)[b, :, :n // 32 * 32], before[b, :, :n // 32 * 32])


@pytest.mark.parametrize("B,H,D,block,cap,cap8,lens", [
    (3, 2, 128, 64, 300, 333, [300, 0, 65]),
    (2, 5, 64, 32, 97, 97, [97, 1]),
    (1, 1, 128, 128, 700, 650, [650]),
])
def test_store_bit_exact(B, H, D, block, cap, cap8, lens):
    rng = np.random.default_rng(cap)
    k, v = _bf16(rng.standard_normal((B, H, cap, D))), _bf16(rng.standard_normal((B, H, cap, D)) * 30)
    for b, n in enumerate(lens):
        k[b, :, n:] = float("nan")
        v[b, :, n:] = float("nan")
    src = sd.KVCache(k, v, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    c = _cache(rng, B, H, cap8, D, block, lens=[7] * B)
    before = c.k.view(torch.uint8).clone()
    sd.kv8_store(c, src)
    assert c.len.tolist() == lens and sd.get_device_error() == 0
    for b, n in enumerate(lens):
        if n:
            for x, t, s in ((k, c.k, c.k_scale), (v, c.v, c.v_scale)):
                nb = -(-n // block)
                codes, scales = oracle.kv8_append(np.zeros((1, H, n, D)), np.ones((1, H, nb)), [0],
                                                  to64(x[b:b + 1, :, :n]).transpose(0, 2, 1, 3), block)
                assert np.array_equal(_codes(t)[b, :, :n], codes[0])
                assert np.array_equal(s.cpu().numpy()[b, :, :nb], scales[0].astype(np.float32))
        assert torch.equal(c.k.view(torch.uint8)[b, :, n:], before[b, :, n:])


def test_store_bad_lengths():
    rng = np.random.default_rng(8)
    k = _bf16(rng.standard_normal((3, 1, 100, 64)))
    c = _cache(rng, 3, 1, 80, 64, 32, lens=[3, 4, 5])
    sd.kv8_store(c, sd.KVCache(k, k.clone(), torch.tensor([101, 81, 80], dtype=torch.int32, device="cuda")))
    assert sd.get_device_error() == sd.SD_DEVERR_KV_OVERFLOW | sd.SD_DEVERR_LENGTH
    assert c.len.tolist() == [3, 4, 80]


# ------------------------------------------------------------------ attention

def _attention_ok(out, q, c, block_mask=False, scale=None):
    """Against the oracle on the dequantised cache. The bound: the output's rounding to
    bf16 (2^-8 |o|), one relative 2^-8 a weight (8 bits of it are kept) and, for weights
    below the smallest normal number of an 8-bit term, 2^-13 of the largest a key, added
    as random errors."""
    lens = c.len.cpu().numpy()
    k = oracle.dequantise(_codes(c.k), c.k_scale.cpu().numpy().astype(np.float64), c.block)
    v = oracle.dequantise(_codes(c.v), c.v_scale.cpu().numpy().astype(np.float64), c.block)
    R = q.shape[1]
    for b, n in enumerate(lens):  # rows that no query sees may hold anything
        k[b, :, n:], v[b, :, n:] = 0.0, 0.0
    kw = {} if scale is None else {"scale": scale}
    ref = oracle.verify_attention(to64(q), k, v, lens, block=block_mask, **kw)
    mag = oracle.verify_attention(to64(q), k, np.abs(v), lens, block=block_mask, **kw)
    top = np.abs(v).max(axis=(1, 2, 3))[:, None, None, None]
    tol = 2.0 ** -8 * np.abs(ref) + 2.0 ** -8 * mag + 2.0 ** -13 * np.sqrt(lens.max() + R) * top * mag.max() / np.maximum(top, mag.max())
    err = np.abs(to64(out) - ref)
    assert np.all(err <= tol), (err.max(), (err - tol).max())
    assert sd.get_device_error() == 0
    return ref


CASES = [
    # D, block, cap, R, Hq, Hkv, lens (with the new rows): decode rows, odd groups, lengths around tiles and blocks
    (128, 64, 300, 1, 4, 1, [1, 2, 127, 128, 129, 300]),
    (128, 64, 700, 8, 32, 8, [8, 9, 640, 641, 700]),
    (128, 32, 4113, 5, 28, 4, [4113, 5, 1000]),
    (64, 32, 1200, 6, 28, 4, [6, 1200, 129]),
    (64, 128, 515, 1, 5, 5, [1, 64, 515]),
    (128, 128, 2100, 17, 32, 8, [2100, 17]),
    (128, 64, 520, 16, 16, 2, [520, 16, 144]),
    (64, 64, 2050, 32, 4, 1, [2050, 33]),
    (128, 64, 300, 128, 2, 2, [300, 128, 131]),
    (64, 64, 400, 100, 1, 1, [100, 399]),
]


@pytest.mark.parametrize("D,block,cap,R,Hq,Hkv,lens", CASES)
@pytest.mark.parametrize("block_mask", [False, True])
def test_attention_parity(D, block, cap, R, Hq, Hkv, lens, block_mask):
    rng = np.random.default_rng(cap + R)
    c = _cache(rng, len(lens), Hkv, cap, D, block, lens=lens)
    for b, n in enumerate(lens):  # stale rows and the scales of blocks past the length
        c.k.view(torch.uint8)[b, :, n:] = 0x7f
        c.v.view(torch.uint8)[b, :, n:] = 0xff
        c.k_scale[b, :, -(-n // block):] = float("nan")
        c.v_scale[b, :, -(-n // block):] = float("inf")
    q = _bf16(rng.standard_normal((len(lens), R, Hq, D)))
    out = torch.full_like(q, float("nan"))
    _attention_ok(sd.kv8_attention(q, c, out=out, block=block_mask), q, c, block_mask)


@pytest.mark.parametrize("spread", [0.0, 8.0, 40.0])
def test_attention_score_range(spread):
    """Scores that all tie, and scores over tens and hundreds of units, the largest late or
    early in the keys; an explicit scale."""
    rng = np.random.default_rng(11)
    c = _cache(rng, 2, 2, 1500, 128, 64, lens=[1500, 1111])
    q = _bf16(rng.standard_normal((2, 7, 8, 128)) * spread)
    _attention_ok(sd.kv8_attention(q, c), q, c)
    c.k_scale.copy_(c.k_scale * torch.linspace(0.1, 2.0, c.k_scale.shape[-1], device="cuda"))
    _attention_ok(sd.kv8_attention(q, c, scale=0.05), q, c, scale=0.05)
    c.k_scale.copy_(c.k_scale.flip(-1))
    c.k_scale[:, :, 1] *= 0.37  # not a power of two
    _attention_ok(sd.kv8_attention(q, c, scale=0.05), q, c, scale=0.05)


def test_attention_rows_of_unlike_magnitude():
    """Rows of one tile from 2^-20 to 2^20: each row is as exact as if it were alone."""
    rng = np.random.default_rng(12)
    c = _cache(rng, 1, 1, 600, 128, 64, lens=[600])
    x = rng.standard_normal((1, 8, 4, 128)) * 2.0 ** rng.integers(-20, 3, (1, 8, 4, 1))
    x[0, 3, 1] = 0.0
    q = _bf16(x)
    _attention_ok(sd.kv8_attention(q, c), q, c)
    c.k_scale *= 2.0 ** -20
    q = _bf16(x * 2.0 ** 20)
    _attention_ok(sd.kv8_attention(q, c), q, c)


def test_attention_value_scales_far_apart():
    rng = np.random.default_rng(13)
    c = _cache(rng, 1, 2, 900, 128, 64, lens=[900])
    for lo in (-20, 0, 20):
        c.v_scale.copy_(torch.from_numpy((2.0 ** (lo + rng.integers(-4, 5, c.v_scale.shape))).astype(np.float32)))
        q = _bf16(rng.standard_normal((1, 8, 8, 128)))
        _attention_ok(sd.kv8_attention(q, c), q, c)


def test_attention_bad_lengths_and_other_scenes():
    rng = np.random.default_rng(14)
    c = _cache(rng, 3, 2, 200, 128, 64, lens=[4, 150, 201])
    q = _bf16(rng.standard_normal((3, 5, 4, 128)))
    out = torch.full_like(q, 3.0)
    sd.kv8_attention(q, c, out=out)
    assert sd.get_device_error() == sd.SD_DEVERR_LENGTH
    assert (out[0] == 3.0).all() and (out[2] == 3.0).all() and not (out[1] == 3.0).all()


def test_attention_is_deterministic_and_follows_the_stream():
    rng = np.random.default_rng(15)
    c = _cache(rng, 4, 4, 3000, 128, 64, lens=[3000, 2000, 1000, 10])
    q = _bf16(rng.standard_normal((4, 8, 16, 128)))
    first = sd.kv8_attention(q, c).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            assert torch.equal(sd.kv8_attention(q, c), first)
    torch.cuda.synchronize()


def test_step_in_a_graph():
    """append, attention, rollback captured once and replayed: the serving loop's use."""
    rng = np.random.default_rng(16)
    c = _cache(rng, 2, 2, 500, 128, 64, lens=[300, 411])
    q, k, v = (_bf16(rng.standard_normal((2, 5, h, 128))) for h in (8, 2, 2))
    keep = torch.tensor([5, 5], dtype=torch.int32, device="cuda")
    none = torch.zeros_like(keep)
    out = torch.empty_like(q)

    def step():
        sd.kv8_append(c, k, v)
        sd.kv8_attention(q, c, out=out)
        sd.kv_rollback(c.len, none, 5)
    step()
    want = out.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    out.zero_()
    for _ in range(3):
        g.replay()
    assert torch.equal(out, want) and c.len.tolist() == [300, 411] and sd.get_device_error() == 0
    sd.kv8_append(c, k, v)
    sd.kv_rollback(c.len, keep, 5)
    assert c.len.tolist() == [305, 416]
    _attention_ok(sd.kv8_attention(q, c), q, c)
