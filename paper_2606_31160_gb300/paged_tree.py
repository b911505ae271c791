"""Verify steps of drafted trees over a paged cache: the paged append, the tree attention,
the acceptance along a tree and the commit used together, on a few layers of a seeded
synthetic target.

A scene's prefix lies in pages that the layers share by one table. Every step drafts a
tree behind the last committed token; a layer rotates the tree's rows and writes their
keys and values into the pages (`sd.paged_append`), and each row attends to the prefix and
its own ancestors (`sd.tree_attention`). The target's logits then pick a path
(`sd.accept_tree`), and its rows move together behind the prefix in every layer's cache
(`sd.paged_commit`).

Trees are accepted greedily only, and the command fills the prefix with random rows: the
attention of a prompt's own rows would go in calls of up to 256 rows, a chain each.

    python -m paper_2606_31160_gb300.paged_tree [--prefix 1000 --nodes 26 --steps 4]
"""

import argparse

import torch

from . import sd


class PagedTreeTarget:
    """The caches of `layers` layers, every scene with pages of its own for `cap` rows, and
    the workspaces of a step of up to `nodes` rows."""

    def __init__(self, layers, B, Hkv, cap, D, nodes, V, page=64, device="cuda"):
        first = sd.PagedKVCache.empty(B, Hkv, cap, D, page=page, device=device)
        self.caches = [first] + [sd.PagedKVCache(torch.zeros_like(first.k), torch.zeros_like(first.v), first.table,
                                                 torch.zeros_like(first.len)) for _ in range(layers - 1)]
        self.group = sd.PagedKVCacheGroup(self.caches)
        self.ws = sd.workspace(sd.accept_tree_workspace_bytes(B, nodes, V), device)

    def attend(self, layer, qkv, heads, pos, sections, parents, n_new=None, interleaved=0, base=1e6):
        """One layer's rows: qkv [B, R, Hq + 2 Hkv, D], a projection's output (read only), heads
        = (Hq, Hkv), pos [B, R, 3]. Returns [B, R, Hq, D]."""
        Hq, Hkv = heads
        q, k, v = qkv.split([Hq, Hkv, Hkv], dim=2)
        q = sd.paged_append(self.caches[layer], k, v, q=q, pos=pos, sections=sections, interleaved=interleaved, base=base,
                            n_new=n_new, q_out=torch.empty(q.shape, dtype=q.dtype, device=q.device))
        return sd.tree_attention(q, self.caches[layer], parents=parents, n_new=n_new)

    def commit(self, logits, tokens, parents, n_new=None):
        """The path that the logits [B, R, V] agree with, kept in every layer. Returns (n_emit
        [B], path [B, R], out [B, R]): the committed rows and the tokens that they emit, then -1."""
        n_emit, path, out, _ = sd.accept_tree(logits, tokens, parents, n_new=n_new, ws=self.ws)
        sd.paged_commit(self.group, path, n_emit, n_new=n_new)
        return n_emit, path, out


def depths(parents):
    """Rows between each row and the prefix, [B, R]: its position is the prefix's length plus
    that. Parents of rows that do not count may be anything: one that is not an earlier row is
    not followed."""
    parents = torch.where(parents < torch.arange(parents.shape[1], device=parents.device), parents, -1)
    at, depth = parents, torch.zeros_like(parents)
    while bool((at >= 0).any()):
        depth += (at >= 0).to(depth.dtype)
        at = torch.where(at >= 0, parents.gather(1, at.clamp_min(0).long()), at)
    return depth


def random_tree(B, R, generator, device="cuda"):
    """Parents of trees whose rows each follow the one before or any earlier one."""
    i = torch.arange(R, device=device)
    any_ = (torch.rand((B, R), generator=generator, device=device) * i).floor().to(torch.int32)
    chain = torch.rand((B, R), generator=generator, device=device) < 0.4
    parents = torch.where(chain, (i - 1).to(torch.int32), any_)
    parents[:, 0] = -1
    return parents


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--prefix", type=int, default=1000)
    ap.add_argument("--nodes", type=int, default=26)
    ap.add_argument("--steps", type=int, default=4)
    ap.add_argument("--scenes", type=int, default=2)
    ap.add_argument("--layers", type=int, default=2)
    a = ap.parse_args(argv)
    B, R, Hq, Hkv, D, V, sections = a.scenes, a.nodes, 32, 8, 128, 151936, (16, 24, 24)
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    target = PagedTreeTarget(a.layers, B, Hkv, a.prefix + (a.steps + 1) * R, D, R, V)
    at = torch.arange(a.prefix, dtype=torch.int32, device="cuda")[None, :, None].expand(B, -1, 3).contiguous()
    for cache in target.caches:  # the prompt
        sd.paged_append(cache, rand(B, a.prefix, Hkv, D), rand(B, a.prefix, Hkv, D), pos=at, sections=sections)
    next_pos = torch.full((B, 1), a.prefix, dtype=torch.int32, device="cuda")
    total = 0
    for step in range(a.steps):
        parents = random_tree(B, R, g)
        pos = (next_pos + depths(parents))[..., None].expand(-1, -1, 3).contiguous()
        for layer in range(a.layers):
            target.attend(layer, rand(B, R, Hq + 2 * Hkv, D), (Hq, Hkv), pos, sections, parents)
        logits = rand(B, R, V) * 2.0  # in a model, of the layers above
        best = logits.argmax(-1).to(torch.int32)
        right = torch.rand((B, R), generator=g, device="cuda") < 0.7
        tokens = torch.where(right, best.gather(1, parents.clamp_min(0).long()), 0)
        n_emit, path, out = target.commit(logits, tokens, parents)
        next_pos += n_emit[:, None]
        total += int(n_emit.sum())
        print("step %d: committed %s of %d rows, paths %s" % (
            step, n_emit.tolist(), R, [path[b, :n].tolist() for b, n in enumerate(n_emit.tolist())]))
    bits = sd.get_device_error()
    if bits:
        raise RuntimeError("device error bits 0x%x" % bits)
    for cache in target.caches:
        if int(cache.len.sum()) != B * a.prefix + total:
            raise RuntimeError("lengths %s" % cache.len.tolist())
    return 0


if __name__ == "__main__":
    raise SystemExit(main())
