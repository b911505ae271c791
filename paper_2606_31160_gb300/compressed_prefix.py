"""Verify steps over a compressed prefix: the 8-bit cache, the eviction and the token
log probabilities used together, one layer of a seeded synthetic target.

A scene's prefix is prefilled into a bf16 cache. The last `window` rows of the prompt
say which of its keys matter: the weight they give each key is accumulated
(`sd.attention_weights`), each KV head keeps the `keep` keys that hold most of it
(`sd.kv_evict`), and what is kept is stored in 8 bits (`sd.kv8_store`). Every verify
step then rotates its rows, appends them (`sd.kv8_append`), attends
(`sd.kv8_attention`), accepts drafts greedily, rolls the cache back to what was
committed, and scores the committed tokens with the entropy and alternatives of their
rows (`sd.token_logprobs`).

    python -m paper_2606_31160_gb300.compressed_prefix [--prefix 4096 --keep 1024 --steps 4]
"""

import argparse

import torch

from . import sd


class CompressedPrefix:
    """One layer's small cache, made from its prefilled bf16 cache (`sd.KVCache`).

    q_window [B, R, Hq, D] bf16, rotated: the last R rows of the prompt, whose keys are
    in the cache. keep: keys of the prompt that each KV head keeps; sinks and recent:
    the first and last ones among them whatever their weight; room: rows to come."""

    def __init__(self, cache, q_window, keep, sinks=4, recent=64, room=128, block=64):
        B, Hkv, _, D = cache.shape
        dev = cache.k.device
        self.weights = sd.attention_weights(q_window, cache)
        kept = sd.KVCache.empty(B, Hkv, keep, D, device=dev)
        self.kept = torch.empty((B, Hkv, keep), dtype=torch.int32, device=dev)
        sd.kv_evict(cache, self.weights, kept, keep, sinks=sinks, recent=recent, kept=self.kept)
        self.cache = sd.KV8Cache.empty(B, Hkv, keep + room, D, block=block, device=dev)
        sd.kv8_store(self.cache, kept)

    def bytes(self):
        """Device bytes of the cache: codes and scales."""
        c = self.cache
        return sum(t.numel() * t.element_size() for t in (c.k, c.v, c.k_scale, c.v_scale))

    def attend(self, q, k_new, v_new, pos, sections, interleaved=0, base=1e6, out=None):
        """sd.verify_layer on the small cache: rotation of q and k_new in place, append,
        attention. Returns out [B, R, Hq, D]."""
        sd.rope_apply(q, k_new, pos, sections, interleaved, base)
        sd.kv8_append(self.cache, k_new, v_new)
        return sd.kv8_attention(q, self.cache, out=out)

    def commit(self, logits, draft, temperature=1.0, top_n=5):
        """Greedy acceptance of draft [B, K] int32 over logits [B, K+1, V], the rollback to
        the committed rows and the committed tokens' scores. Returns (n_emit, tokens,
        logprob, entropy, top_ids, top_logprobs); tokens past n_emit are -1, their
        logprob 0, so a scene's sum is the log probability of what it committed."""
        n_emit, tokens, _ = sd.accept_greedy(logits, draft)
        sd.kv_rollback(self.cache.len, n_emit, logits.shape[1])
        return (n_emit, tokens) + sd.token_logprobs(logits, tokens, temperature=temperature, top_n=top_n)


def synthetic_prompt(B, L, Hq, Hkv, D, window, seed=0, device="cuda"):
    """A prefilled cache in which some keys are what the prompt's last rows look at:
    (cache, q_window)."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    k = torch.randn((B, Hkv, L, D), generator=g, device=device)
    v = torch.randn((B, Hkv, L, D), generator=g, device=device)
    q = torch.randn((B, window, Hq, D), generator=g, device=device)
    heavy = torch.randperm(L, generator=g, device=device)[:max(1, L // 16)]
    mean = q.view(B, window, Hkv, Hq // Hkv, D).mean((1, 3))
    k[:, :, heavy] += 4.0 * mean[:, :, None] * D ** 0.5 / mean.norm(dim=-1)[:, :, None, None]
    lens = torch.full((B,), L, dtype=torch.int32, device=device)
    return sd.KVCache(k.to(torch.bfloat16), v.to(torch.bfloat16), lens), q.to(torch.bfloat16)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--prefix", type=int, default=4096)
    ap.add_argument("--keep", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=4)
    ap.add_argument("--scenes", type=int, default=2)
    a = ap.parse_args(argv)
    B, Hq, Hkv, D, K, V, window = a.scenes, 32, 8, 128, 7, 151936, 32
    sections = (16, 24, 24)
    cache, q_window = synthetic_prompt(B, a.prefix, Hq, Hkv, D, window)
    small = CompressedPrefix(cache, q_window, a.keep, room=a.steps * (K + 1) + K + 1)
    mass = small.weights.sum(-1, keepdim=True)
    share = (small.weights.gather(2, small.kept.long().clamp_min(0)).sum(-1, keepdim=True) / mass).mean().item()
    print("prefix %d -> %d keys a head in 8 bits: %.2f -> %.2f MB, %.1f%% of the window's attention weight kept" % (
        a.prefix, a.keep, 2 * cache.k.numel() * 2 / 1e6, small.bytes() / 1e6, 100 * share))
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    next_pos = torch.full((B,), a.prefix, dtype=torch.int32, device="cuda")
    for step in range(a.steps):
        pos = (next_pos[:, None] + torch.arange(K + 1, dtype=torch.int32, device="cuda"))[..., None].expand(-1, -1, 3).contiguous()
        small.attend(rand(B, K + 1, Hq, D), rand(B, K + 1, Hkv, D), rand(B, K + 1, Hkv, D), pos, sections)
        logits = rand(B, K + 1, V) * 2.0  # in a model, of the layers above
        draft = torch.where(torch.rand((B, K), generator=g, device="cuda") < 0.6, logits[:, :K].argmax(-1), 0).to(torch.int32)
        n_emit, tokens, logprob, entropy, top_ids, top_logprobs = small.commit(logits, draft)
        next_pos += n_emit
        print("step %d: committed %s, log probability %s, mean entropy %.2f nats, best alternative %s" % (
            step, n_emit.tolist(), ["%.2f" % x for x in logprob.sum(-1).tolist()], entropy.mean().item(), top_ids[0, 0, 1].item()))
    bits = sd.get_device_error()
    if bits:
        raise RuntimeError("device error bits 0x%x" % bits)
    return 0


if __name__ == "__main__":
    raise SystemExit(main())
