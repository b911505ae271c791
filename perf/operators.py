"""Operators that make a long prefix small and score what the target answers, as
measurable cases:

  * the 8-bit KV cache: appending a verify step's rows (`kv8_append`) and storing a
    whole bf16 cache (`kv8_store`), with one scale for each block of tokens, KV head
    and scene; and the verify attention that reads it (`kv8_attention`);
  * the attention weight that each cached key accumulates (`attention_weights`) and
    the eviction of the keys that hold least of it (`kv_evict`);
  * the log probabilities of given tokens with the entropy and the top alternatives
    of their rows (`token_logprobs`).

Each case has a plain form in elementary torch operations and, where `own` is set,
the call that a user makes. Sizes are those of the repository's workloads: 32 query /
8 KV heads x 128 (target), 16 / 4 x 128 (draft), 28 / 4 x 64, prefixes of up to 16384
keys, K up to 16 drafts, a vocabulary of 151936. `draw` spreads over the same ranges,
with odd batch sizes, group sizes, prefixes and vocabularies.

Layouts: cache [B, Hkv, capacity, D], its lengths [B] int32, scales
[B, Hkv, ceil(capacity / block)] fp32, new rows [B, R, Hkv, D], queries [B, R, Hq, D],
key weights [B, Hkv, capacity] fp32, logits [B, R, V].
"""

import math

import numpy as np
import torch

own = False

DEV = "cuda"
E4M3_MAX = 448.0
MIN_EXP = -100  # smallest scale: 2^-100


def listed():
    return [
        # a verify step's new rows of one target layer into the 8-bit cache, one scene:
        # the smallest call, all latency
        dict(name="kv8_append_step", kind="append", B=1, R=8, Hkv=8, D=128, L=4096, block=64),
        # a prefilled bf16 cache of four scenes stored in 8 bits: all bandwidth
        dict(name="kv8_store_prefix", kind="store", B=4, Hkv=8, D=128, L=16384, block=64),
        # plain decoding of the draft: a single row a step
        dict(name="kv8_attention_decode", kind="attention", B=1, R=1, Hq=16, Hkv=4, D=128, L=4096, block=64, mask="causal"),
        # one scene's verify rows of one target layer
        dict(name="kv8_attention_step", kind="attention", B=1, R=8, Hq=32, Hkv=8, D=128, L=4096, block=64, mask="causal"),
        # batched serving: 32 ragged scenes, K = 8
        dict(name="kv8_attention_b32", kind="attention", B=32, R=9, Hq=32, Hkv=8, D=128, L=8192, block=64, mask="causal"),
        # head dim 64, seven query heads a KV head, an odd batch and capacity, small blocks
        dict(name="kv8_attention_d64", kind="attention", B=5, R=6, Hq=28, Hkv=4, D=64, L=4099, block=32, mask="causal"),
        # the weights that a verify step's committed rows give to the keys of one layer
        dict(name="weights_step", kind="weights", B=1, R=8, Hq=32, Hkv=8, D=128, L=4096, committed="some"),
        # an observation window of 32 rows at the end of eight ragged prefixes
        dict(name="weights_window", kind="weights", B=8, R=32, Hq=32, Hkv=8, D=128, L=8192, committed="all"),
        # one scene's layer down to half its keys
        dict(name="evict_step", kind="evict", B=1, Hkv=8, D=128, L=4096, keep=2048, sinks=4, recent=64),
        # eight ragged long prefixes down to 4096 keys each
        dict(name="evict_batch", kind="evict", B=8, Hkv=8, D=128, L=16384, keep=4096, sinks=4, recent=256),
        # one scene's verify rows: the committed tokens' scores, five alternatives
        dict(name="logprobs_step", kind="logprobs", B=1, R=8, V=151936, dtype="bf16", top_n=5, temperature=1.0, masked=False),
        # a batch's rows in fp32, part of the vocabulary masked out, twenty alternatives
        dict(name="logprobs_batch", kind="logprobs", B=32, R=8, V=151936, dtype="f32", top_n=20, temperature=0.6, masked=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# bytes and operations of a drawn pass stay below those of its kind's largest listed case
_MOST = {"append": 3.4e8, "store": 3.4e8, "attention": 4.6e8, "weights": 1.2e8, "evict": 2.6e8, "logprobs": 1.5e8}
_MOST_FLOPS = {"attention": 3.3e10, "weights": 1.4e10}


def draw(rng):
    kind = rng.choice(["append", "store", "attention", "attention", "weights", "evict", "logprobs"])
    Hq, Hkv, D = rng.choice([(32, 8, 128), (16, 4, 128), (28, 4, 128), (8, 8, 128), (28, 4, 64), (4, 1, 64), (16, 4, 64)])
    while True:
        B, L = _log_int(rng, 1, 32), _log_int(rng, 200, 16384)
        if kind == "append":
            c = dict(kind=kind, B=B, R=_log_int(rng, 1, 500), Hkv=Hkv, D=D, L=L, block=rng.choice([32, 64, 128]))
        elif kind == "store":
            c = dict(kind=kind, B=B, Hkv=Hkv, D=D, L=L, block=rng.choice([32, 64, 128]))
        elif kind == "attention":
            c = dict(kind=kind, B=B, R=rng.randint(1, 17), Hq=Hq, Hkv=Hkv, D=D, L=L, block=rng.choice([32, 64, 128]),
                     mask=rng.choice(["causal", "causal", "causal", "block"]))
            if Hq // Hkv * c["R"] > 128:
                continue
        elif kind == "weights":
            c = dict(kind=kind, B=min(B, 8), R=_log_int(rng, 1, 32), Hq=Hq, Hkv=Hkv, D=D, L=L, committed=rng.choice(["some", "all"]))
        elif kind == "evict":
            c = dict(kind=kind, B=B, Hkv=Hkv, D=D, L=L, keep=0, sinks=rng.randint(0, 8), recent=0)
            c["keep"] = max(16, int(L * rng.uniform(0.1, 0.9)))
            c["recent"] = min(rng.randint(0, 256), (c["keep"] - c["sinks"]) // 2)
        else:
            c = dict(kind=kind, B=B, R=rng.randint(1, 17), V=rng.choice([4096, 32000, 50257, 128256, 151936, 151936]),
                     dtype=rng.choice(["bf16", "bf16", "f32"]), top_n=rng.randint(0, 20),
                     temperature=rng.choice([1.0, 0.6, 1.3]), masked=rng.random() < 0.3)
        if work(c)["bytes"] <= _MOST[kind] and work(c)["flops"] <= _MOST_FLOPS.get(kind, math.inf):
            return c


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + 12345) & 0x7FFFFFFF)
    return g


def _lengths(case):
    """Keys cached per scene: L for a single scene, U[0.75 L, L] for a batch (a
    property of the workload: every seed's batch is equally ragged)."""
    B, L = case["B"], case["L"]
    if B == 1:
        return np.array([L], dtype=np.int32)
    return np.random.RandomState(1000 + 31 * B + L).randint(-(-3 * L // 4), L + 1, size=B).astype(np.int32)


def _capacity(case):
    """Room for the prefix, 17 new rows (or the case's own) and nothing else."""
    return case["L"] + max(17, case["R"] if case["kind"] == "append" else 0)


def _rows(g, *shape):
    """Keys or values as projections give them: normal, with a few channels of a head
    several times larger than the rest."""
    x = torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)
    return x * (1.0 + 3.0 * (torch.arange(shape[-1], device=DEV) % 29 == 7)).to(torch.bfloat16)


def _blocks(n, block):
    return -(-n // block)


def _pow2(e):
    """2^e, exact, of an int tensor."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _scale_exp(m, e):
    """Exponent of the smallest power of two s with x <= 448 s, x = m 2^e as frexp gives it."""
    return torch.where(m <= 0.875, e - 9, e - 8)


def _encode(x, scale):
    return (x / scale).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)


def _finite_amax(x, dims):
    a = x.abs()
    return torch.where(a < math.inf, a, torch.zeros_like(a)).amax(dims)


def _fresh_scale(amax):
    m, e = torch.frexp(amax)
    return _pow2(torch.where(amax > 0, _scale_exp(m, e), torch.full_like(e, MIN_EXP)).clamp_min(MIN_EXP))


def _quantised(x, block):
    """A cache's worth of rows [B, H, n, D] as codes and block scales."""
    B, H, n, D = x.shape
    nb = _blocks(n, block)
    y = torch.nn.functional.pad(x.float(), (0, 0, 0, nb * block - n)).view(B, H, nb, block, D)
    s = _fresh_scale(_finite_amax(y, (3, 4)))
    return _encode(y, s[..., None, None]).view(B, H, nb * block, D)[:, :, :n].contiguous(), s


def _kv8(case, g, lens):
    cap = _capacity(case)
    s = {}
    for w in "kv":
        s[w], s[w + "_scale"] = _quantised(_rows(g, case["B"], case["Hkv"], cap, case["D"]), case["block"])
    s["len"] = torch.from_numpy(lens).to(DEV)
    return s


def _kv16(case, g, lens):
    shape = (case["B"], case["Hkv"], _capacity(case), case["D"])
    return dict(k=_rows(g, *shape), v=_rows(g, *shape), len=torch.from_numpy(lens).to(DEV))


def _committed(case):
    """Rows that the acceptance kept, per scene."""
    B, R = case["B"], case["R"]
    if case["committed"] == "all":
        return None
    n = np.random.RandomState(77 + B + R).randint(1, R + 1, size=B).astype(np.int32)
    return torch.from_numpy(n).to(DEV)


def prepare(case, seed):
    g = _gen(seed)
    kind, B, D = case["kind"], case["B"], case.get("D")
    s = dict(case=case)
    if kind in ("append", "store", "attention", "weights", "evict"):
        lens = _lengths(case)
        cap = _capacity(case)
    if kind == "append":
        s.update(_kv8(case, g, lens))
        s["len0"] = s["len"].clone()
        s["k_new"] = _rows(g, B, case["R"], case["Hkv"], D)
        s["v_new"] = _rows(g, B, case["R"], case["Hkv"], D)
    elif kind == "store":
        s.update(_kv16(case, g, lens))
        nb = _blocks(cap, case["block"])
        for w in "kv":
            s[w + "8"] = torch.zeros(s["k"].shape, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
            s[w + "8_scale"] = torch.zeros((B, case["Hkv"], nb), device=DEV)
        s["len8"] = torch.zeros(B, dtype=torch.int32, device=DEV)
    elif kind == "attention":
        s.update(_kv8(case, g, lens + case["R"] if B == 1 else np.maximum(lens, case["R"])))
        s["q"] = torch.randn((B, case["R"], case["Hq"], D), generator=g, device=DEV, dtype=torch.bfloat16)
        s["out"] = torch.zeros_like(s["q"])
    elif kind == "weights":
        s.update(_kv16(case, g, np.maximum(lens, case["R"])))
        del s["v"]
        s["q"] = torch.randn((B, case["R"], case["Hq"], D), generator=g, device=DEV, dtype=torch.bfloat16)
        s["committed"] = _committed(case)
        s["weights_in"] = torch.rand((B, case["Hkv"], cap), generator=g, device=DEV)
        s["weights"] = torch.zeros_like(s["weights_in"])
    elif kind == "evict":
        s.update(_kv16(case, g, lens))
        keep, H = case["keep"], case["Hkv"]
        # accumulated weights: most keys hold little, some exactly nothing (ties)
        w = torch.randn((B, H, cap), generator=g, device=DEV).mul_(2.0).exp_()
        s["weights"] = torch.where(torch.rand(w.shape, generator=g, device=DEV) < 0.3, torch.zeros_like(w), w)
        s["k2"] = torch.zeros((B, H, keep + 17, D), dtype=torch.bfloat16, device=DEV)
        s["v2"] = torch.zeros_like(s["k2"])
        s["len2"] = torch.zeros(B, dtype=torch.int32, device=DEV)
        s["weights2"] = torch.zeros((B, H, keep + 17), device=DEV)
        s["kept"] = torch.zeros((B, H, keep), dtype=torch.int32, device=DEV)
    else:
        R, V, n = case["R"], case["V"], case["top_n"]
        dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        z = torch.randn((B, R, V), generator=g, device=DEV).mul_(2.0).to(dt)
        if case["masked"]:  # tokens that a grammar or a mask forbids
            z[..., torch.rand(V, generator=g, device=DEV) < 0.3] = -math.inf
        tokens = torch.randint(0, V, (B, R), generator=g, device=DEV)
        top = torch.rand((B, R), generator=g, device=DEV) < 0.6  # most are what the model expects
        tokens = torch.where(top, z.argmax(-1), tokens).to(torch.int32)
        past = torch.rand(B, generator=g, device=DEV) < 0.4  # the last rows were not committed
        tokens[:, -1] = torch.where(past, torch.full_like(tokens[:, -1], -1), tokens[:, -1])
        s.update(logits=z, tokens=tokens, logprob=torch.zeros((B, R), device=DEV), entropy=torch.zeros((B, R), device=DEV),
                 top_ids=torch.zeros((B, R, n), dtype=torch.int32, device=DEV), top_logprobs=torch.zeros((B, R, n), device=DEV))
    if own:
        _handles(s)
    return s


def _handles(s):
    """The cache handles that a program keeps beside its tensors."""
    from paper_2606_31160_gb300 import sd
    kind = s["case"]["kind"]
    s["sd"] = sd
    if kind in ("append", "attention"):
        s["cache8"] = sd.KV8Cache(s["k"], s["v"], s["k_scale"], s["v_scale"], s["len"], s["case"]["block"])
    elif kind == "store":
        s["cache"] = sd.KVCache(s["k"], s["v"], s["len"])
        s["cache8"] = sd.KV8Cache(s["k8"], s["v8"], s["k8_scale"], s["v8_scale"], s["len8"], s["case"]["block"])
    elif kind == "weights":
        s["cache"] = sd.KVCache(s["k"], s["k"], s["len"])
    elif kind == "evict":
        s["cache"] = sd.KVCache(s["k"], s["v"], s["len"])
        s["cache2"] = sd.KVCache(s["k2"], s["v2"], s["len2"])


# ------------------------------------------------------------------ one pass

def run(s):
    kind = s["case"]["kind"]
    if kind == "append":
        s["len"].copy_(s["len0"])  # the committed lengths that the loop hands over
    if own:
        _own_pass(s, kind)
    else:
        _PLAIN[kind](s)
    return {name: s[name] for name in _OUTPUTS[kind]}


_OUTPUTS = {
    "append": ("k", "v", "k_scale", "v_scale", "len"),
    "store": ("k8", "v8", "k8_scale", "v8_scale", "len8"),
    "attention": ("out",),
    "weights": ("weights",),
    "evict": ("k2", "v2", "len2", "weights2", "kept"),
    "logprobs": ("logprob", "entropy", "top_ids", "top_logprobs"),
}


def _own_pass(s, kind):
    sd, c = s["sd"], s["case"]
    if kind == "append":
        sd.kv8_append(s["cache8"], s["k_new"], s["v_new"])
    elif kind == "store":
        sd.kv8_store(s["cache8"], s["cache"])
    elif kind == "attention":
        sd.kv8_attention(s["q"], s["cache8"], out=s["out"], block=c["mask"] == "block")
    elif kind == "weights":
        sd.attention_weights(s["q"], s["cache"], weights_in=s["weights_in"], weights=s["weights"], decay=0.9,
                             committed=s["committed"])
    elif kind == "evict":
        sd.kv_evict(s["cache"], s["weights"], s["cache2"], c["keep"], sinks=c["sinks"], recent=c["recent"],
                    weights_out=s["weights2"], kept=s["kept"])
    else:
        sd.token_logprobs(s["logits"], s["tokens"], temperature=c["temperature"], top_n=c["top_n"], logprob=s["logprob"],
                          entropy=s["entropy"], top_ids=s["top_ids"], top_logprobs=s["top_logprobs"])


def _plain_append(s):
    """New rows into the blocks that they touch. A block that begins with them takes
    its scale from them; a block that holds older rows keeps its scale times the least
    power of two (1 or more) that fits them, and its older codes follow."""
    c = s["case"]
    B, R, block, cap = c["B"], c["R"], c["block"], s["k"].shape[2]
    W = (R - 1) // block + 2
    n0 = s["len0"].long()
    first = n0 // block
    p = first[:, None] * block + torch.arange(W * block, device=DEV)  # [B, W * block]
    new = (p >= n0[:, None]) & (p < n0[:, None] + R)
    at = p.clamp_max(cap - 1)  # repeated at the cache's end, with the same values
    wb = at // block - first[:, None]
    blk = (first[:, None] + torch.arange(W, device=DEV)).clamp_max(_blocks(cap, block) - 1)
    held = (first[:, None] + torch.arange(W, device=DEV)) * block < n0[:, None]  # older rows in the block
    any_new = new.view(B, W, block).any(-1)
    row = (p - n0[:, None]).clamp(0, R - 1)
    row_at = (at - n0[:, None]).clamp(0, R - 1)
    is_new = ((at >= n0[:, None]) & (at < n0[:, None] + R))[:, None, :, None]
    is_old = (at < n0[:, None])[:, None, :, None]
    bi = torch.arange(B, device=DEV)[:, None]
    for w in "kv":
        codes, scale = s[w].view(torch.uint8), s[w + "_scale"]
        x = s[w + "_new"].float()
        amax = torch.where(new[:, :, None, None], x[bi, row], torch.zeros((), device=DEV))
        amax = _finite_amax(amax.view(B, W, block, -1, c["D"]), (2, 4)).transpose(1, 2)  # [B, H, W]
        old = scale[bi, :, blk].transpose(1, 2)
        m, e = torch.frexp(amax.double() / old.double())
        grow = torch.where(amax > 0, _scale_exp(m, e), torch.zeros_like(e)).clamp_min(0)
        held_, any_ = held[:, None], any_new[:, None]
        # (2^grow may pass fp32 where a block held nothing but zeros: in 64 bits)
        grown = (old.double() * torch.pow(2.0, grow.double())).float()
        s_new = torch.where(any_, torch.where(held_, grown, _fresh_scale(amax)), old)
        shrink = _pow2(-torch.where(held_ & any_, grow, torch.zeros_like(grow)).clamp_max(60))
        per = wb[:, None].expand(-1, c["Hkv"], -1)
        old_rows = codes[bi, :, at].view(torch.float8_e4m3fn).transpose(1, 2).float()  # [B, H, W * block, D]
        moved = (old_rows * shrink.gather(2, per)[..., None]).to(torch.float8_e4m3fn)
        moved = torch.where(is_old, moved.view(torch.uint8), old_rows.to(torch.float8_e4m3fn).view(torch.uint8))
        fresh = _encode(x[bi, row_at].transpose(1, 2), s_new.gather(2, per)[..., None])
        codes[bi, :, at] = torch.where(is_new, fresh.view(torch.uint8), moved).transpose(1, 2)
        last = _blocks(cap, block) - 1 - first  # windows past the cache's end repeat its last block
        s_at = s_new.gather(2, torch.arange(W, device=DEV)[None].minimum(last[:, None])[:, None].expand(-1, c["Hkv"], -1))
        scale[bi, :, blk] = s_at.transpose(1, 2)
    s["len"].copy_(s["len0"] + R)


def _plain_store(s):
    c = s["case"]
    block, cap = c["block"], s["k"].shape[2]
    valid = torch.arange(cap, device=DEV) < s["len"][:, None]
    nb = _blocks(cap, block)
    full = torch.arange(nb, device=DEV) * block < s["len"][:, None]
    for w in "kv":
        codes, scale = _quantised(torch.where(valid[:, None, :, None], s[w].float(), torch.zeros((), device=DEV)), block)
        out, out_scale = s[w + "8"].view(torch.uint8), s[w + "8_scale"]
        out.copy_(torch.where(valid[:, None, :, None], codes.view(torch.uint8), out))
        out_scale.copy_(torch.where(full[:, None], scale, out_scale))
    s["len8"].copy_(s["len"])


def _softmax_weights(q, k, lens, block_mask):
    """exp(score - max) and its sum over the keys that each row sees: [B, Hkv, G, R, n], [..., 1]."""
    B, R, Hq, D = q.shape
    Hkv, n = k.shape[1], k.shape[2]
    qg = q.float().view(B, R, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, D)
    z = (qg @ k.transpose(2, 3)).view(B, Hkv, Hq // Hkv, R, n) * (1.0 / math.sqrt(D))
    last = lens.long()[:, None] - R + torch.arange(R, device=DEV)
    if block_mask:
        last = (lens.long()[:, None] - 1).expand(B, R)
    seen = torch.arange(n, device=DEV) <= last[..., None]
    z = z.masked_fill(~seen[:, None, None], -math.inf)
    e = torch.exp(z - z.amax(-1, keepdim=True))
    return e, e.sum(-1, keepdim=True)


def _plain_attention(s):
    c = s["case"]
    cap, block = s["k"].shape[2], c["block"]
    of = torch.arange(cap, device=DEV) // block
    k = s["k"].float() * s["k_scale"][..., of][..., None]
    v = s["v"].float() * s["v_scale"][..., of][..., None]
    e, total = _softmax_weights(s["q"], k, s["len"], c["mask"] == "block")
    B, Hkv, G, R, n = e.shape
    o = (e.view(B, Hkv, G * R, n) @ v).view(B, Hkv, G, R, -1) / total
    s["out"].copy_(o.permute(0, 3, 1, 2, 4).reshape(s["out"].shape))


def _plain_weights(s):
    c = s["case"]
    e, total = _softmax_weights(s["q"], s["k"].float(), s["len"], False)
    p = e / total
    if s["committed"] is not None:
        p = p * (torch.arange(c["R"], device=DEV) < s["committed"][:, None])[:, None, None, :, None]
    n = torch.arange(p.shape[-1], device=DEV)
    lens = s["len"][:, None, None]
    before = torch.where(n < lens - c["R"], 0.9 * s["weights_in"], torch.zeros((), device=DEV))
    s["weights"].copy_(torch.where(n < lens, before + p.sum((2, 3)), s["weights"]))


def _plain_evict(s):
    c = s["case"]
    keep, cap = c["keep"], s["k"].shape[2]
    lens = s["len"].long()[:, None, None]
    n = torch.arange(cap, device=DEV)
    w = torch.where((n < c["sinks"]) | (n >= lens - c["recent"]), torch.full((), math.inf, device=DEV), s["weights"])
    w = torch.where(n < lens, w, torch.full((), -1.0, device=DEV))  # (accumulated weights are not negative)
    best = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :keep]
    count = lens.clamp_max(keep)
    some = torch.arange(keep, device=DEV) < count
    kept = torch.sort(torch.where(some, best, torch.full((), cap, device=DEV)), dim=-1).values
    some = some.expand_as(kept)
    at = torch.where(some, kept, torch.zeros_like(kept))
    s["kept"].copy_(torch.where(some, kept, torch.full((), -1, device=DEV)))
    for w_ in "kv":
        rows = s[w_].gather(2, at[..., None].expand(-1, -1, -1, c["D"]))
        s[w_ + "2"][:, :, :keep] = torch.where(some[..., None], rows, s[w_ + "2"][:, :, :keep])
    s["weights2"][:, :, :keep] = torch.where(some, s["weights"].gather(2, at), s["weights2"][:, :, :keep])
    s["len2"].copy_(s["len"].clamp_max(keep))


def _plain_logprobs(s):
    c = s["case"]
    z = s["logits"].float() + 0.0  # (-0 and +0 are equal)
    x = (z - z.amax(-1, keepdim=True)) / c["temperature"]
    e = torch.exp(x)
    total = e.sum(-1)
    ln = torch.log(total)
    s["entropy"].copy_(ln - torch.where(e > 0, e * x, torch.zeros((), device=DEV)).sum(-1) / total)
    t = s["tokens"].long()
    lp = x.gather(-1, t.clamp_min(0)[..., None])[..., 0] - ln
    s["logprob"].copy_(torch.where(t >= 0, lp, torch.zeros_like(lp)))
    if c["top_n"]:
        bits = z.view(torch.int32).long()
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)
        key = (order << 32) - torch.arange(c["V"], device=DEV)  # equal values: the lowest index first
        ids = torch.topk(key, c["top_n"], dim=-1).indices
        s["top_ids"].copy_(ids)
        s["top_logprobs"].copy_(x.gather(-1, ids) - ln[..., None])


_PLAIN = {"append": _plain_append, "store": _plain_store, "attention": _plain_attention, "weights": _plain_weights,
          "evict": _plain_evict, "logprobs": _plain_logprobs}


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    c = case
    B, D = c["B"], c.get("D", 0)
    if c["kind"] == "logprobs":
        rows = B * c["R"]
        elem = 2 if c["dtype"] == "bf16" else 4
        return {"bytes": rows * (c["V"] * elem + 12 + 8 * c["top_n"]), "flops": 5 * rows * c["V"]}
    keys = float(_lengths(c).sum())
    if c["kind"] == "append":
        n = B * c["R"] * c["Hkv"]
        return {"bytes": 2 * n * D * 3 + 8 * B, "flops": 4 * n * D}
    if c["kind"] == "store":
        n = keys * c["Hkv"]
        return {"bytes": 2 * n * (3 * D + 4.0 / c["block"]), "flops": 4 * n * D}
    if c["kind"] == "evict":
        kept = float(np.minimum(_lengths(c), c["keep"]).sum())
        return {"bytes": c["Hkv"] * (4 * keys + kept * (8 * D + 8)), "flops": c["Hkv"] * keys}
    if B == 1 and c["kind"] == "attention":
        keys += c["R"]
    rows = B * c["R"] * c["Hq"] * D
    pairs = c["Hq"] * c["R"] * keys
    if c["kind"] == "attention":
        return {"bytes": 2 * keys * c["Hkv"] * (D + 4.0 / c["block"]) + 4 * rows, "flops": 4 * pairs * D}
    return {"bytes": keys * c["Hkv"] * (2 * D + 8) + 2 * rows, "flops": 2 * pairs * D}


# ------------------------------------------------------------------ the definitions in 64 bits

def _round_e4m3(x):
    """The nearest e4m3 value (ties to even) of float64 |x| <= 448, by its binade."""
    e = torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -20))).clamp_min(-6)
    step = torch.exp2(e - 3)
    step = torch.where(x.abs() >= 16 * step, 2 * step, step)  # log2 rounded down at a power of two
    return (torch.round(x / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def _exact_block(rows, old_codes, old_scale):
    """One block of one head: its new rows beside its older codes (0 rows: a fresh block)."""
    amax = float(rows.abs().max()) if rows.numel() else 0.0
    if old_codes.shape[0] == 0:
        scale = 2.0 ** MIN_EXP
        if amax > 0:
            e = max(MIN_EXP, math.frexp(amax / E4M3_MAX)[1] - 1)
            scale = 2.0 ** (e + (amax > E4M3_MAX * 2.0 ** e))
    else:
        scale = old_scale
        while amax > E4M3_MAX * scale:
            scale *= 2.0
        old_codes = _round_e4m3(old_codes * (old_scale / scale))
    return torch.cat([old_codes, _round_e4m3(rows / scale)]), scale


def _exact_append(s, c):
    out = {}
    n0s = s["len"].tolist()
    for w in "kv":
        codes, scales = s[w].double().clone(), s[w + "_scale"].double().clone()
        new = s[w + "_new"].double()
        for b in range(c["B"]):
            n0, end = n0s[b], n0s[b] + c["R"]
            for blk in range(n0 // c["block"], (end - 1) // c["block"] + 1):
                lo, hi = blk * c["block"], min((blk + 1) * c["block"], end)
                first = max(lo, n0)
                for h in range(c["Hkv"]):
                    codes[b, h, lo:hi], scales[b, h, blk] = _exact_block(
                        new[b, first - n0:hi - n0, h], codes[b, h, lo:first], float(scales[b, h, blk]))
        out[w], out[w + "_scale"] = codes, scales
    out["len"] = s["len"] + c["R"]
    return out


def _exact_store(s, c):
    out = {"len8": s["len"].clone()}
    for w in "kv":
        x = s[w].double()
        codes, scales = torch.zeros_like(x), torch.zeros_like(s[w + "8_scale"], dtype=torch.float64)
        for b, n in enumerate(s["len"].tolist()):
            for lo in range(0, n, c["block"]):
                hi = min(lo + c["block"], n)
                amax = x[b, :, lo:hi].abs().amax((1, 2))
                sc = torch.exp2(torch.ceil(torch.log2((amax / E4M3_MAX).clamp_min(2.0 ** MIN_EXP))))
                sc = torch.where(amax <= E4M3_MAX * sc / 2, sc / 2, torch.where(amax > E4M3_MAX * sc, 2 * sc, sc))
                codes[b, :, lo:hi] = _round_e4m3(x[b, :, lo:hi] / sc[:, None, None])
                scales[b, :, lo // c["block"]] = sc
        out[w + "8"], out[w + "8_scale"] = codes, scales
    return out


def _exact_rows(s, c, b, h, k):
    """Softmax of scene b's rows of query head h over keys k [len, D] in 64 bits: [R, len]."""
    n = k.shape[0]
    z = s["q"][b, :, h].double() @ k.T / math.sqrt(c["D"])
    for i in range(c["R"]):
        if c.get("mask") != "block":
            z[i, n - c["R"] + i + 1:] = -math.inf
    return torch.softmax(z, -1)


def _exact_attention(s, c):
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    for b, n in enumerate(s["len"].tolist()):
        for g in range(c["Hkv"]):
            rep = lambda t: t[b, g].double().repeat_interleave(c["block"])[:n, None]  # noqa: E731
            k, v = s["k"][b, g, :n].double() * rep(s["k_scale"]), s["v"][b, g, :n].double() * rep(s["v_scale"])
            for h in range(g * c["Hq"] // c["Hkv"], (g + 1) * c["Hq"] // c["Hkv"]):
                out[b, :, h] = _exact_rows(s, c, b, h, k) @ v
    return {"out": out}


def _exact_weights(s, c):
    out = torch.zeros(s["weights"].shape, dtype=torch.float64, device=DEV)
    for b, n in enumerate(s["len"].tolist()):
        rows = c["R"] if s["committed"] is None else int(s["committed"][b])
        for g in range(c["Hkv"]):
            acc = s["weights_in"][b, g, :n].double() * 0.9
            acc[n - c["R"]:] = 0.0
            k = s["k"][b, g, :n].double()
            for h in range(g * c["Hq"] // c["Hkv"], (g + 1) * c["Hq"] // c["Hkv"]):
                acc += _exact_rows(s, c, b, h, k)[:rows].sum(0)
            out[b, g, :n] = acc
    return {"weights": out}


def _exact_logprobs(s, c):
    z = s["logits"].double() / c["temperature"]
    lp = torch.log_softmax(z, -1)
    t = s["tokens"].long()
    at = lp.gather(-1, t.clamp_min(0)[..., None])[..., 0]
    p = lp.exp()
    h = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(-1)
    return {"logprob": torch.where(t >= 0, at, torch.zeros_like(at)), "entropy": h, "top_ids": None,
            "top_logprobs": torch.topk(lp, c["top_n"], dim=-1).values}


def exact(case, seed):
    """The outputs that are computed numbers, in 64 bits, from the definitions, scene
    by scene (indices and rows that an eviction moves have no value but the plain form's)."""
    global own
    kind = case["kind"]
    if kind == "evict" or (kind == "append" and case["B"] * case["R"] * case["Hkv"] > 20000):
        return None
    if kind == "store" and float(_lengths(case).sum()) / case["block"] > 20000:
        return None
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    with torch.no_grad():
        got = {"append": _exact_append, "store": _exact_store, "attention": _exact_attention, "weights": _exact_weights,
               "logprobs": _exact_logprobs}[kind](s, case)
    return {k: (v.cpu() if v is not None else None) for k, v in got.items()}
