"""The compressed prefix end to end: window weights, eviction, 8-bit cache, verify steps
and scores, against the same steps on the oracle."""
import numpy as np
import pytest
import torch

import oracle
from paper_2606_31160_gb300 import compressed_prefix, sd
from tests.helpers import ensure_lib, to64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_lib()
    sd.get_device_error()


def test_steps_against_the_oracle():
    B, L, Hq, Hkv, D, W, K, V, keep = 2, 600, 8, 2, 128, 16, 3, 5000, 200
    cache, qw = compressed_prefix.synthetic_prompt(B, L, Hq, Hkv, D, W)
    small = compressed_prefix.CompressedPrefix(cache, qw, keep, sinks=2, recent=8, room=40)
    w64 = oracle.attention_weights(to64(qw), to64(cache.k), [L] * B)
    got = small.weights.cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got - w64) <= 2e-5 * w64 + 1e-6 * W * Hq / Hkv)
    codes = {"k": np.zeros((B, Hkv, keep + 40, D)), "v": np.zeros((B, Hkv, keep + 40, D))}
    scales = {n: np.ones((B, Hkv, -(-(keep + 40) // 64))) for n in "kv"}
    for h in range(Hkv):
        for b in range(B):  # the kernel's own weights decide: nothing near a tie may move
            want = oracle.kept_keys(got[b, h], L, keep, 2, 8)
            assert small.kept[b, h].tolist() == want.tolist()
    for n, t in (("k", cache.k), ("v", cache.v)):
        rows = np.stack([to64(t)[b][np.arange(Hkv)[:, None], small.kept[b].cpu().numpy()] for b in range(B)])
        codes[n], scales[n] = oracle.kv8_append(codes[n], scales[n], [0] * B, rows.transpose(0, 2, 1, 3), 64)
    lens, rng = np.array([keep] * B), np.random.default_rng(3)
    for step in range(3):
        bf = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(torch.bfloat16).cuda()  # noqa: E731
        q, k, v = bf(B, K + 1, Hq, D), bf(B, K + 1, Hkv, D), bf(B, K + 1, Hkv, D)
        pos = torch.from_numpy((L + 4 * step + np.arange(K + 1))[None, :, None].repeat(B, 0).repeat(3, 2).astype(np.int32)).cuda()
        out = small.attend(q, k, v, pos, (16, 24, 24))
        for n, x in (("k", k), ("v", v)):  # k: rotated in place
            codes[n], scales[n] = oracle.kv8_append(codes[n], scales[n], lens, to64(x), 64)
        assert np.array_equal(small.cache.k.float().cpu().numpy(), codes["k"])
        ref = oracle.verify_attention(to64(q), *(oracle.dequantise(codes[n], scales[n], 64) for n in "kv"), lens + K + 1)
        # the output's rounding and 8-bit weights (2^-8 each) on values of up to about 4
        assert np.all(np.abs(to64(out) - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -6)
        logits = bf(B, K + 1, V)
        draft = logits[:, :K].argmax(-1).to(torch.int32)
        draft[:, 1 + step % 2] += 1
        n_emit, tokens, logprob, entropy, ids, _ = small.commit(logits, draft)
        lens = lens + n_emit.cpu().numpy()
        assert small.cache.len.tolist() == lens.tolist() and n_emit.tolist() == [2 + step % 2] * B
        rl, rh, ri, _ = oracle.token_logprobs(to64(logits).reshape(-1, V), tokens.cpu().numpy().reshape(-1), 1.0, 5)
        assert np.abs(to64(logprob).reshape(-1) - rl).max() <= 1e-5 and np.abs(to64(entropy).reshape(-1) - rh).max() <= 1e-5
        assert np.array_equal(ids.cpu().numpy().reshape(-1, 5), ri)
    assert sd.get_device_error() == 0


def test_command_runs(capsys):
    assert compressed_prefix.main(["--prefix", "1024", "--keep", "256", "--steps", "2"]) == 0
    assert "step 1: committed" in capsys.readouterr().out
