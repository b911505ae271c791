"""Attention over the 8-bit cache where one key holds most of a row's weight and a long
tail the rest: the tail's mass and its values stay, wherever the key lies."""
import numpy as np
import pytest
import torch

import oracle
from paper_2606_31160_gb300 import sd, workloads
from tests.helpers import attn_within, ensure_lib, to64

pytestmark = pytest.mark.gpu

SHARES = (0.3, 0.5, 0.6, 0.7, 0.8, 0.9, 0.95, 0.99)  # of the key that stands out, a row each
PLACES = ("first", "middle", "last")                 # its tile, a KV head each
R, G = 2, 4
SCALE = 2.0 ** -7


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_lib()
    sd.get_device_error()
    yield
    sd.set_cluster_size(0)


def _scene(rng, n, D, tail):
    """Codes [Hkv, n, D] of the keys, query rows [R, Hq, D] and the keys that stand out."""
    H = len(PLACES)
    k = np.zeros((H, n, D))
    q = np.zeros((R, H * G, D))
    if tail == "lognormal":
        k[..., 1:] = oracle.round_e4m3(np.clip(rng.standard_normal((H, n, D - 1)) * 100, -448, 448))
        q[..., 1:] = rng.standard_normal((R, H * G, D - 1)) * 1.6
    peaks = [5, n // 2 + 3, n - 3]
    for h, j in enumerate(peaks):
        k[h, j] = 0.0
        k[h, j, 0] = 448.0
    q = workloads.to_bf16(q.astype(np.float32)).float().numpy().astype(np.float64)
    for i in range(R):
        for h in range(H * G):
            z = k[h // G] @ q[i, h] * SCALE / np.sqrt(D)
            rest = np.exp(z).sum() - np.exp(z[peaks[h // G]])
            share = SHARES[i * G + h % G]
            q[i, h, 0] = np.log(share / (1 - share) * rest) * np.sqrt(D) / (448 * SCALE)
    return k, workloads.to_bf16(q.astype(np.float32)), peaks


def _cache(k, v, B):
    H, n, D = k.shape
    c = sd.KV8Cache.empty(B, H, n, D, 64)
    for t, x in ((c.k, k), (c.v, v)):
        t.copy_(torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).cuda()[None].view(torch.uint8)
                .expand(B, -1, -1, -1).contiguous().view(torch.float8_e4m3fn))
    c.k_scale.fill_(SCALE)
    c.v_scale.fill_(SCALE)
    c.len.fill_(n)
    return c


def _tolerance(q, k, v, ref):
    """The output's rounding (2^-9 of it, doubled), six standard deviations of the weights'
    roundings (8 significant bits: 2^-9 / sqrt 3 of each; of the small ones half a step of
    2^-13 where the row's sum is 2^7 or more: 2^-21 of it), as random errors over the keys."""
    n, D = k.shape[1], k.shape[2]
    tol = np.empty_like(ref)
    for i in range(R):
        for h in range(ref.shape[1]):
            g = h // G
            z = k[g, :n - R + i + 1] @ q[i, h] / np.sqrt(D)
            p = np.exp(z - z.max())
            p /= p.sum()
            x = v[g, :len(p)] ** 2
            tol[i, h] = 2.0 ** -8 * np.abs(ref[i, h]) + 6 * 2.0 ** -9 / np.sqrt(3) * np.sqrt(p ** 2 @ x) + \
                6 * 2.0 ** -21 * np.sqrt(x.sum(0))
    return tol


@pytest.mark.parametrize("shape", ["one CTA a head", "clusters", "even shares"])
@pytest.mark.parametrize("tail", ["flat", "lognormal"])
@pytest.mark.parametrize("n", [4096, 8192, 16384])
@pytest.mark.parametrize("D", [64, 128])
def test_one_key_over_a_long_tail(D, n, tail, shape):
    rng = np.random.default_rng(n + D)
    H = len(PLACES)
    k, q, peaks = _scene(rng, n, D, tail)
    B = 1
    if shape == "even shares":
        B = next(b for b in range(16, 128) if sd.kv8_attention_workspace_bytes(b, R, H * G, H, D, n) > 0)
    sd.set_cluster_size(1 if shape == "one CTA a head" else 0)
    try:
        qd = q.cuda()[None].expand(B, -1, -1, -1).contiguous()
        out = to64(sd.kv8_attention(qd, _cache(k, np.full_like(k, 128.0), B)))
        # all values 1: 2^-9 for the weights, 2^-9 for the output
        assert np.abs(out - 1.0).max() <= 2.0 ** -8, (out.min(), out.max())
        v = oracle.round_e4m3(np.clip(rng.standard_normal(k.shape) * 100, -448, 448))
        for h, j in enumerate(peaks):  # the key that stands out has a small value
            v[h, j] = oracle.round_e4m3(v[h, j] * 0.05)
        out = to64(sd.kv8_attention(qd, _cache(k, v, B)))
    finally:
        sd.set_cluster_size(0)
    k, v, q = k * SCALE, v * SCALE, to64(q)
    ref = oracle.verify_attention(q[None], k[None], v[None], [n])[0]
    assert attn_within(out, ref[None])
    err = np.abs(out - ref) - _tolerance(q, k, v, ref)
    assert err.max() <= 0, err.max()
    assert sd.get_device_error() == 0


@pytest.mark.parametrize("shape", ["one CTA a head", "clusters"])
@pytest.mark.parametrize("D", [64, 128])
def test_four_keys_alike_over_a_long_tail(D, shape):
    """One in each 32 of the first tile's keys, together 0.3 to 0.99 of the row."""
    rng = np.random.default_rng(D)
    n, at = 16384, [5, 40, 70, 100]
    k, q, peaks = _scene(rng, n, D, "flat")
    for h, j in enumerate(peaks):
        k[h, j] = 0.0
        k[h, at, 0] = 448.0
    q = to64(q)
    for i in range(R):
        for h in range(len(PLACES) * G):
            share = SHARES[i * G + h % G]
            q[i, h, 0] = np.log(share / (1 - share) * (n - 4) / 4) * np.sqrt(D) / (448 * SCALE)
    q = workloads.to_bf16(q.astype(np.float32))
    sd.set_cluster_size(1 if shape == "one CTA a head" else 0)
    try:
        out = to64(sd.kv8_attention(q.cuda()[None], _cache(k, np.full_like(k, 128.0), 1)))
        assert np.abs(out - 1.0).max() <= 2.0 ** -8, (out.min(), out.max())
        v = oracle.round_e4m3(np.clip(rng.standard_normal(k.shape) * 100, -448, 448))
        v[:, at] = oracle.round_e4m3(v[:, at] * 0.05)
        out = to64(sd.kv8_attention(q.cuda()[None], _cache(k, v, 1)))
    finally:
        sd.set_cluster_size(0)
    k, v, q = k * SCALE, v * SCALE, to64(q)
    ref = oracle.verify_attention(q[None], k[None], v[None], [n])[0]
    # half a step of 2^-13 where the row's sum is 2^3 or more
    tol = _tolerance(q, k, v, ref) + 6 * 2.0 ** -17 * np.sqrt((v ** 2).sum(1)).repeat(G, 0)
    assert np.all(np.abs(out - ref) <= tol), (np.abs(out - ref) - tol).max()
    assert attn_within(out, ref[None])
    assert sd.get_device_error() == 0
