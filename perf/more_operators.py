"""Verifying a tree of drafted tokens over a paged KV cache, as measurable cases:

  * appending new rows to a paged cache, the keys rotated on the way and the queries
    beside them (`paged_append`);
  * the attention of a drafted tree's rows over such a cache: a row sees the prefix and
    its own ancestors (`tree_attention`);
  * greedy acceptance along a tree: the longest path that the target agrees with, and
    the token that follows it (`accept_tree`);
  * the commit of what was accepted: the path's rows move together, in every layer's
    cache, and the lengths follow (`paged_commit`).

Each case has a plain form in elementary torch operations and, where `own` is set,
the call that a user makes. Heads, head dims, prefixes and the vocabulary are those of
the repository's workloads (32 query / 8 KV heads x 128, 16 / 4 x 128, 28 / 4 x 64, up
to 16384 keys, 151936 tokens) and one generic long cache. `draw` spreads over the same
ranges, with odd batch sizes, tree sizes, prefixes and pages.

Layouts: pools [pages, Hkv, page, D], page table [B, max_pages] int32, lengths [B]
int32, new rows [B, R, Hkv, D], queries [B, R, Hq, D] (the append's may be parts of one
projection's output [B, R, Hq + 2 Hkv, D]), parents [B, R] int32 (-1: the row follows the
prefix; otherwise an earlier row), rows that count [B] int32, logits [B, R, V].
"""

import math

import numpy as np
import torch

own = False

DEV = "cuda"
SECTIONS = {128: (16, 24, 24), 64: (8, 12, 12)}
BASE = 1e6


def listed():
    return [
        # a verify step's rows of one target layer, one scene: the smallest call, all latency
        dict(name="append_step", kind="append", B=1, R=8, Hq=32, Hkv=8, D=128, L=4096, page=64, fused=True, ragged=False,
             interleaved=0, vision=False),
        # chunks of four prompts, vision patches among them: all bandwidth
        dict(name="append_prompt", kind="append", B=4, R=2048, Hq=32, Hkv=8, D=128, L=4096, page=64, fused=True, ragged=False,
             interleaved=0, vision=True),
        # ragged trees of a batch, head dim 64, small pages, interleaved axes
        dict(name="append_ragged", kind="append", B=32, R=61, Hq=28, Hkv=4, D=64, L=4099, page=16, fused=False, ragged=True,
             interleaved=1, vision=False),
        # plain decoding of the draft: a single row a step
        dict(name="attention_decode", kind="attention", B=1, R=1, Hq=16, Hkv=4, D=128, L=4096, page=16, tree=False, ragged=False),
        # one scene's drafted tree of 25 tokens behind the last committed one
        dict(name="attention_step", kind="attention", B=1, R=26, Hq=32, Hkv=8, D=128, L=4096, page=64, tree=True, ragged=False),
        # batched serving: 32 ragged scenes, trees of 60 drafted tokens
        dict(name="attention_b32", kind="attention", B=32, R=61, Hq=32, Hkv=8, D=128, L=8192, page=64, tree=True, ragged=False),
        # head dim 64, seven query heads a KV head, odd sizes, ragged trees
        dict(name="attention_d64", kind="attention", B=5, R=13, Hq=28, Hkv=4, D=64, L=4099, page=32, tree=True, ragged=True),
        # a chain of eight rows over one very long cache
        dict(name="attention_long", kind="attention", B=1, R=8, Hq=32, Hkv=8, D=128, L=131072, page=128, tree=False,
             ragged=False),
        # one scene's tree against the target's logits
        dict(name="accept_step", kind="accept", B=1, R=26, V=151936, dtype="bf16", ragged=False),
        # a batch's ragged trees against fp32 logits
        dict(name="accept_batch", kind="accept", B=16, R=61, V=151936, dtype="f32", ragged=True),
        # what one scene accepted, in all 36 layers' caches
        dict(name="commit_step", kind="commit", layers=36, B=1, R=26, Hkv=8, D=128, L=4096, page=64, ragged=False),
        # what a batch accepted, in all 36 layers' caches
        dict(name="commit_batch", kind="commit", layers=36, B=32, R=61, Hkv=8, D=128, L=500, page=16, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# bytes and operations of a drawn pass stay below those of its kind's largest listed case
_MOST = {"append": 2.0e8, "attention": 1.0e9, "accept": 3.2e8, "commit": 1.8e7}
_MOST_FLOPS = {"attention": 2.2e11}


def draw(rng):
    kind = rng.choice(["append", "append", "attention", "attention", "attention", "attention", "accept", "commit"])
    Hq, Hkv, D = rng.choice([(32, 8, 128), (16, 4, 128), (28, 4, 128), (8, 8, 128), (28, 4, 64), (4, 1, 64), (16, 4, 64)])
    page = rng.choice([16, 32, 64, 128])
    ragged = rng.random() < 0.4
    while True:
        B = _log_int(rng, 1, 32)
        if kind == "append":
            c = dict(kind=kind, B=B, R=_log_int(rng, 1, 2048), Hq=Hq, Hkv=Hkv, D=D, L=_log_int(rng, 16, 8192), page=page,
                     fused=rng.random() < 0.5, ragged=ragged, interleaved=rng.randint(0, 1), vision=rng.random() < 0.5)
        elif kind == "attention":
            c = dict(kind=kind, B=B, R=_log_int(rng, 1, 128), Hq=Hq, Hkv=Hkv, D=D, L=_log_int(rng, 16, 131072), page=page,
                     tree=rng.random() < 0.7, ragged=ragged)
        elif kind == "accept":
            c = dict(kind=kind, B=B, R=_log_int(rng, 1, 128), V=rng.choice([4096, 32000, 50257, 128256, 151936, 151936]),
                     dtype=rng.choice(["bf16", "bf16", "f32"]), ragged=ragged)
        else:
            c = dict(kind=kind, layers=rng.randint(1, 36), B=B, R=_log_int(rng, 2, 128), Hkv=Hkv, D=D,
                     L=_log_int(rng, 16, 2048), page=page, ragged=ragged)
            if c["layers"] * B * (c["L"] + c["R"]) * Hkv * D > 8e8:  # the pools fit beside one another
                continue
        if work(c)["bytes"] <= _MOST[kind] and work(c)["flops"] <= _MOST_FLOPS.get(kind, math.inf):
            return c


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + 54321) & 0x7FFFFFFF)
    return g


def _lengths(case):
    """Keys cached per scene before the new rows: L for a single scene, U[0.75 L, L] for a
    batch (a property of the workload: every seed's batch is equally ragged)."""
    B, L = case["B"], case["L"]
    if B == 1:
        return np.array([L], dtype=np.int32)
    return np.random.RandomState(2000 + 31 * B + L).randint(-(-3 * L // 4), L + 1, size=B).astype(np.int32)


def _counts(case):
    """New rows per scene: R, or U[1, R] where the batch's trees differ in size."""
    B, R = case["B"], case["R"]
    if not case["ragged"]:
        return np.full(B, R, dtype=np.int32)
    n = np.random.RandomState(3000 + 17 * B + R).randint(1, R + 1, size=B)
    n[0] = R
    return n.astype(np.int32)


def _tree(rs, R, deepest=10):
    """Parents of a drafted tree in the order that the nodes were added: some extend the
    node before, others branch off earlier; row 0 is the last committed token."""
    parents, depth = [-1], [0]
    for i in range(1, R):
        p = i - 1 if rs.rand() < 0.35 else rs.randint(0, i)
        while depth[p] >= deepest:
            p = parents[p]
        parents.append(p)
        depth.append(depth[p] + 1)
    return parents, depth


def _trees(case, seed):
    rs = np.random.RandomState((int(seed) * 7919 + case["R"]) & 0x7FFFFFFF)
    both = [_tree(rs, case["R"]) for _ in range(case["B"])]
    return np.array([p for p, _ in both], dtype=np.int32), np.array([d for _, d in both], dtype=np.int32), rs


def _walk(rs, parents, n):
    """A path from row 0 down through random children, to a random end."""
    kids = [[] for _ in range(n)]
    for i in range(1, n):
        kids[parents[i]].append(i)
    path = [0]
    while kids[path[-1]] and rs.rand() < 0.8:
        path.append(kids[path[-1]][rs.randint(len(kids[path[-1]]))])
    return path


def _paths(case):
    """Accepted paths and their lengths (a property of the workload). A pass can be repeated
    on the same pools: no row that a path keeps is moved over."""
    parents, _, rs = _trees(case, 5)
    counts = _counts(case)
    path = np.full((case["B"], case["R"]), -1, dtype=np.int32)
    n_emit = np.zeros(case["B"], dtype=np.int32)
    for b in range(case["B"]):
        for _ in range(50):
            p = _walk(rs, parents[b], counts[b])
            while any(i != r and i in p for i, r in enumerate(p)):
                p = p[:-1]
            if len(p) > n_emit[b]:
                path[b, :len(p)], n_emit[b] = p, len(p)
            if n_emit[b] >= min(4, counts[b]):
                break
    return path, n_emit


def _rows(g, *shape):
    """Keys or values as projections give them: normal, with a few channels of a head
    several times larger than the rest."""
    x = torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)
    return x * (1.0 + 3.0 * (torch.arange(shape[-1], device=DEV) % 29 == 7)).to(torch.bfloat16)


def _pages(case):
    """Pages a scene: its longest prefix and its new rows."""
    return -(-(case["L"] + case["R"]) // case["page"])


def _pool(case, g, layers=None):
    """Pools with every scene's pages in a random order, a few pages spare, and the table."""
    B, per = case["B"], _pages(case)
    n = B * per + 3
    shape = (n, case["Hkv"], case["page"], case["D"])
    if layers is not None:
        shape = (layers,) + shape
    table = torch.randperm(n, generator=g, device=DEV)[:B * per].view(B, per).to(torch.int32)
    return dict(k=_rows(g, *shape), v=_rows(g, *shape), table=table)


def _on(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def prepare(case, seed):
    g = _gen(seed)
    kind, B, R = case["kind"], case["B"], case["R"]
    counts = _counts(case)
    s = dict(case=case, n_new=_on(counts) if case["ragged"] else None)
    if kind == "append":
        s.update(_pool(case, g))
        lens = _lengths(case)
        s["len0"] = _on(lens)
        s["len"] = s["len0"].clone()
        Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
        if case["fused"]:
            s["q"], s["k_new"], s["v_new"] = _rows(g, B, R, Hq + 2 * Hkv, D).split([Hq, Hkv, Hkv], dim=2)
        else:
            s["q"], s["k_new"], s["v_new"] = _rows(g, B, R, Hq, D), _rows(g, B, R, Hkv, D), _rows(g, B, R, Hkv, D)
        s["q_out"] = torch.zeros((B, R, Hq, D), dtype=torch.bfloat16, device=DEV)
        at = lens[:, None] + np.arange(R)
        if case["vision"]:  # patches of cameras on 28 x 32 grids
            pos = np.stack([at // 896, at // 32 % 28, at % 32], -1)
        else:
            pos = np.repeat(at[..., None], 3, -1)
        s["pos"] = _on(pos.astype(np.int32))
    elif kind == "attention":
        s.update(_pool(case, g))
        s["len"] = _on(_lengths(case) + counts)
        s["q"] = torch.randn((B, R, case["Hq"], case["D"]), generator=g, device=DEV, dtype=torch.bfloat16)
        s["parents"] = _on(_trees(case, seed)[0]) if case["tree"] else None
        s["out"] = torch.zeros_like(s["q"])
    elif kind == "accept":
        dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        parents, _, rs = _trees(case, seed)
        z = torch.randn((B, R, case["V"]), generator=g, device=DEV, dtype=dt).mul_(2.0)
        tokens = rs.randint(0, case["V"], size=(B, R)).astype(np.int32)
        rows, ids = [], []
        for b in range(B):  # where the target agrees with the draft
            path = _walk(rs, parents[b], counts[b])
            rows += [b * R + i for i in path[:-1]]
            ids += [tokens[b, c] for c in path[1:]]
        if rows:
            z.view(B * R, -1)[_on(np.array(rows)), _on(np.array(ids)).long()] = 16.0
        s.update(logits=z, tokens=_on(tokens), parents=_on(parents))
        i32 = dict(dtype=torch.int32, device=DEV)
        s.update(n_emit=torch.zeros(B, **i32), path=torch.zeros((B, R), **i32), out=torch.zeros((B, R), **i32),
                 argmax=torch.zeros((B, R), **i32))
    else:
        s.update(_pool(case, g, case["layers"]))
        lens = np.tile(_lengths(case) + counts, (case["layers"], 1))
        s["len0"] = _on(lens)
        s["len"] = s["len0"].clone()
        path, n_emit = _paths(case)
        s.update(path=_on(path), n_emit=_on(n_emit))
    if own:
        _handles(s)
    return s


def _handles(s):
    """The handles and workspaces that a program keeps beside its tensors."""
    from paper_2606_31160_gb300 import sd
    c = s["case"]
    s["sd"] = sd
    if c["kind"] in ("append", "attention"):
        s["cache"] = sd.PagedKVCache(s["k"], s["v"], s["table"], s["len"])
    elif c["kind"] == "commit":
        s["group"] = sd.PagedKVCacheGroup([sd.PagedKVCache(s["k"][i], s["v"][i], s["table"], s["len"][i])
                                           for i in range(c["layers"])])
    else:
        s["ws"] = sd.workspace(sd.accept_tree_workspace_bytes(c["B"], c["R"], c["V"]))


# ------------------------------------------------------------------ one pass

def run(s):
    kind = s["case"]["kind"]
    if kind in ("append", "commit"):
        s["len"].copy_(s["len0"])  # the lengths that the loop hands over
    if own:
        _own_pass(s, kind)
    else:
        _PLAIN[kind](s)
    return {name: s[name] for name in _OUTPUTS[kind]}


_OUTPUTS = {
    "append": ("k", "v", "len", "q_out"),
    "attention": ("out",),
    "accept": ("n_emit", "path", "out", "argmax"),
    "commit": ("k", "v", "len"),
}


def _own_pass(s, kind):
    sd, c = s["sd"], s["case"]
    if kind == "append":
        sd.paged_append(s["cache"], s["k_new"], s["v_new"], q=s["q"], pos=s["pos"], sections=SECTIONS[c["D"]],
                        interleaved=c["interleaved"], base=BASE, n_new=s["n_new"], q_out=s["q_out"])
    elif kind == "attention":
        sd.tree_attention(s["q"], s["cache"], parents=s["parents"], n_new=s["n_new"], out=s["out"])
    elif kind == "accept":
        sd.accept_tree(s["logits"], s["tokens"], s["parents"], n_new=s["n_new"], ws=s["ws"], n_emit=s["n_emit"],
                       path=s["path"], out=s["out"], argmax=s["argmax"])
    else:
        sd.paged_commit(s["group"], s["path"], s["n_emit"], n_new=s["n_new"])


def _new_rows(s):
    """Scene and row of every new row that counts."""
    c = s["case"]
    if s["n_new"] is None:
        return (torch.arange(c["B"], device=DEV).repeat_interleave(c["R"]), torch.arange(c["R"], device=DEV).repeat(c["B"]))
    return torch.nonzero(torch.arange(c["R"], device=DEV) < s["n_new"][:, None], as_tuple=True)


def _place(s, b, n):
    """Page and slot of row n of scene b."""
    page = s["case"]["page"]
    return s["table"][b, n // page].long(), n % page


def _rotated(x, pos, c):
    """x [rows, H, D] by its coordinates pos [rows, 3]: adjacent pairs, angles in 64 bits."""
    D = c["D"]
    d = torch.arange(D // 2, device=DEV)
    theta = torch.pow(torch.full((), BASE, dtype=torch.float64, device=DEV), -2.0 * d / D)
    s1, s2, _ = SECTIONS[D]
    axis = d % 3 if c["interleaved"] else (d >= s1).long() + (d >= s1 + s2).long()
    phi = pos[:, axis].double() * theta
    cos, sin = phi.cos().float()[:, None], phi.sin().float()[:, None]
    x = x.float()
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2).to(torch.bfloat16)


def _plain_append(s):
    c = s["case"]
    b, r = _new_rows(s)
    pos = s["pos"][b, r]
    page, slot = _place(s, b, s["len0"].long()[b] + r)
    s["k"][page, :, slot] = _rotated(s["k_new"][b, r], pos, c)
    s["v"][page, :, slot] = s["v_new"][b, r]
    s["q_out"][b, r] = _rotated(s["q"][b, r], pos, c)
    s["len"].copy_(s["len0"] + (c["R"] if s["n_new"] is None else s["n_new"]))


def _ancestors(parents):
    """[B, R, R] truth values: row j is row i or an ancestor of it."""
    B, R = parents.shape
    at = torch.arange(R, device=DEV).expand(B, R)
    seen = torch.zeros((B, R, R + 1), dtype=torch.bool, device=DEV)
    for _ in range(min(R, 12)):  # (the trees are at most ten deep)
        seen.scatter_(2, torch.where(at < 0, torch.full_like(at, R), at)[..., None], True)
        at = torch.where(at < 0, at, parents.long().gather(1, at.clamp_min(0)))
    return seen[..., :R]


def _plain_attention(s):
    c = s["case"]
    B, R, Hq, D = s["q"].shape
    Hkv, page = c["Hkv"], c["page"]
    n = s["table"].shape[1] * page
    k, v = (s[w][s["table"].long()].transpose(1, 2).reshape(B, Hkv, n, D).float() for w in "kv")
    count = torch.full((B,), R, device=DEV) if s["n_new"] is None else s["n_new"].long()
    if s["parents"] is None:
        tree = torch.ones((R, R), dtype=torch.bool, device=DEV).tril().expand(B, R, R)
    else:
        tree = _ancestors(s["parents"])
    at = torch.arange(n, device=DEV)
    prefix = s["len"].long() - count
    j = (at - prefix[:, None]).clamp(0, R - 1)[:, None].expand(B, R, n)
    seen = (at < prefix[:, None])[:, None] | ((at < s["len"][:, None])[:, None] & (at >= prefix[:, None])[:, None]
                                              & tree.gather(2, j))
    q = s["q"].float().view(B, R, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, D)
    z = (q @ k.transpose(2, 3)).view(B, Hkv, Hq // Hkv, R, n) * (1.0 / math.sqrt(D))
    z = z.masked_fill(~seen[:, None, None], -math.inf)
    counted = torch.arange(R, device=DEV) < count[:, None]
    z = torch.where(counted[:, None, None, :, None], z, torch.zeros((), device=DEV))  # (rows that do not count)
    e = torch.exp(z - z.amax(-1, keepdim=True))
    o = (e.view(B, Hkv, -1, n) @ v).view(B, Hkv, Hq // Hkv, R, D) / e.sum(-1, keepdim=True)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, R, Hq, D).to(torch.bfloat16)
    s["out"].copy_(torch.where(counted[..., None, None], o, s["out"]))


def _plain_accept(s):
    c = s["case"]
    B, R, V = c["B"], c["R"], c["V"]
    z = s["logits"]
    top = z.amax(-1, keepdim=True)
    best = torch.where(z == top, torch.arange(V, device=DEV, dtype=torch.int32), V).amin(-1)
    count = torch.full((B,), R, device=DEV) if s["n_new"] is None else s["n_new"].long()
    counted = torch.arange(R, device=DEV) < count[:, None]
    s["argmax"].copy_(torch.where(counted, best, s["argmax"]))
    # a row follows its parent where the target agrees, and is the first that does
    p = s["parents"].long().clamp_min(0)
    follows = counted & (s["parents"] >= 0) & (best.gather(1, p) == s["tokens"])
    at = torch.zeros((B, 1), dtype=torch.long, device=DEV)
    path, out = torch.full_like(s["path"], -1), torch.full_like(s["out"], -1)
    emit = torch.zeros((B, 1), dtype=torch.long, device=DEV)
    done = torch.zeros((B, 1), dtype=torch.bool, device=DEV)
    rows = torch.arange(R, device=DEV)
    for i in range(min(R, 12)):
        path[:, i:i + 1] = torch.where(done, path[:, i:i + 1], at.int())
        out[:, i:i + 1] = torch.where(done, out[:, i:i + 1], best.gather(1, at))
        emit += ~done
        nxt = torch.where(follows & (p == at), rows, R).amin(-1, keepdim=True)
        done = done | (nxt == R)
        at = torch.where(done, at, nxt)
    s["path"].copy_(path)
    s["out"].copy_(out)
    s["n_emit"].copy_(emit[:, 0])


def _plain_commit(s):
    c = s["case"]
    R = c["R"]
    count = R if s["n_new"] is None else s["n_new"]
    first = (s["len0"][0] - count).long()
    b, i = torch.nonzero(torch.arange(R, device=DEV) < s["n_emit"][:, None], as_tuple=True)
    src_page, src = _place(s, b, first[b] + s["path"][b, i].long())
    page, slot = _place(s, b, first[b] + i)
    for w in "kv":
        s[w][:, page, :, slot] = s[w][:, src_page, :, src]
    s["len"].copy_(s["len0"] - count + s["n_emit"])


_PLAIN = {"append": _plain_append, "attention": _plain_attention, "accept": _plain_accept, "commit": _plain_commit}


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    c = case
    B, R, D = c["B"], c["R"], c.get("D", 0)
    counts = _counts(c).astype(np.float64)
    rows = float(counts.sum())
    if c["kind"] == "append":
        return {"bytes": rows * (4 * D * (c["Hq"] + 2 * c["Hkv"]) + 12) + 12 * B, "flops": 3 * rows * D * (c["Hq"] + c["Hkv"])}
    if c["kind"] == "accept":
        elem = 2 if c["dtype"] == "bf16" else 4
        return {"bytes": rows * (c["V"] * elem + 12) + 8 * B * R, "flops": rows * c["V"]}
    if c["kind"] == "commit":
        path, n_emit = _paths(c)
        moved = float((path > np.arange(R)).sum())  # rows that are not in their place
        return {"bytes": c["layers"] * (moved * c["Hkv"] * D * 8 + 8 * B) + 4 * float(n_emit.sum()) + 8 * B, "flops": moved}
    keys = _lengths(c) + counts
    q = rows * c["Hq"] * D
    pairs = float((keys * counts).sum()) * c["Hq"]
    return {"bytes": 4 * float(keys.sum()) * (c["Hkv"] * D + 1.0 / c["page"]) + 4 * q + 8 * B + (4 * rows if c["tree"] else 0),
            "flops": 4 * pairs * D}


# ------------------------------------------------------------------ the definitions in 64 bits

def _exact_rotation(x, pos, c):
    """Each pair as a complex number, turned by its angle."""
    D = c["D"]
    half = D // 2
    theta = torch.tensor([BASE ** (-2.0 * d / D) for d in range(half)], dtype=torch.float64, device=DEV)
    if c["interleaved"]:
        axis = [d % 3 for d in range(half)]
    else:
        axis = [a for a, n in enumerate(SECTIONS[D]) for _ in range(n)]
    phi = pos.double()[..., axis] * theta
    z = torch.view_as_complex(x.double().reshape(*x.shape[:-1], half, 2))
    return torch.view_as_real(z * torch.polar(torch.ones_like(phi), phi)[..., None, :]).flatten(-2)


def _exact_append(s, c):
    out = {"k": s["k"].double(), "v": None, "len": None, "q_out": torch.zeros(s["q_out"].shape, dtype=torch.float64, device=DEV)}
    counts = _counts(c)
    for b, n0 in enumerate(s["len0"].tolist()):
        n = int(counts[b])
        turned = _exact_rotation(s["k_new"][b, :n], s["pos"][b, :n], c)
        out["q_out"][b, :n] = _exact_rotation(s["q"][b, :n], s["pos"][b, :n], c)
        first = n0 // c["page"]
        for pg in range(first, (n0 + n - 1) // c["page"] + 1):
            lo, hi = max(n0, pg * c["page"]), min(n0 + n, (pg + 1) * c["page"])
            at = int(s["table"][b, pg])
            out["k"][at, :, lo - pg * c["page"]:hi - pg * c["page"]] = turned[lo - n0:hi - n0].transpose(0, 1)
    return out


def _exact_attention(s, c):
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    counts = _counts(c)
    G = c["Hq"] // c["Hkv"]
    for b, n in enumerate(s["len"].tolist()):
        m = int(counts[b])
        hidden = torch.ones((m, n), dtype=torch.bool, device=DEV)
        hidden[:, :n - m] = False
        if s["parents"] is None:
            up = [i - 1 for i in range(m)]
        else:
            up = s["parents"][b].tolist()
        sees = np.zeros((m, m), dtype=bool)
        for i in range(m):
            if up[i] >= 0:
                sees[i] = sees[up[i]]
            sees[i, i] = True
        hidden[:, n - m:] = ~torch.from_numpy(sees).to(DEV)
        pages = s["table"][b, :-(-n // c["page"])].long()
        for g in range(c["Hkv"]):
            k = s["k"][pages, g].reshape(-1, c["D"])[:n].double()
            v = s["v"][pages, g].reshape(-1, c["D"])[:n].double()
            for h in range(g * G, (g + 1) * G):
                z = s["q"][b, :m, h].double() @ k.T / math.sqrt(c["D"])
                out[b, :m, h] = torch.softmax(z.masked_fill(hidden, -math.inf), -1) @ v
    return {"out": out}


def exact(case, seed):
    """The outputs that are computed numbers, in 64 bits, from the definitions, scene by
    scene (indices and rows that move have no value but the plain form's)."""
    global own
    if case["kind"] in ("accept", "commit"):
        return None
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    with torch.no_grad():
        got = (_exact_append if case["kind"] == "append" else _exact_attention)(s, case)
    return {k: (v.cpu() if v is not None else None) for k, v in got.items()}
