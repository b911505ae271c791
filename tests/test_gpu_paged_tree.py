"""The target of drafted trees over pages (paged_tree.py): a step against the oracle, the
positions of a tree, and the command."""
import numpy as np
import pytest
import torch

import oracle
from helpers import to64
from paper_2606_31160_gb300 import build, paged_tree, sd

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    sd.get_device_error()


def test_depths():
    parents = torch.tensor([[-1, 0, 0, 1, 3, -1], [-1, 0, 1, 2, 3, 4]], dtype=torch.int32, device="cuda")
    assert paged_tree.depths(parents).tolist() == [[0, 1, 1, 2, 3, 0], [0, 1, 2, 3, 4, 5]]


def test_two_steps():
    """What a layer attends to after a commit is what was committed (bound: see test_gpu_tree)."""
    g = torch.Generator(device="cuda").manual_seed(0)
    B, R, Hq, Hkv, D, V, sec = 2, 9, 8, 2, 64, 500, (8, 12, 12)
    target = paged_tree.PagedTreeTarget(2, B, Hkv, 60, D, R, V, page=16)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    lens, kept = [0] * B, [[[np.zeros((0, Hkv, D))] * 2 for _ in range(B)] for _ in range(2)]
    for _ in range(3):
        parents = paged_tree.random_tree(B, R, g)
        pos = (torch.tensor(lens, dtype=torch.int32, device="cuda")[:, None] + paged_tree.depths(parents))[..., None].expand(-1, -1, 3).contiguous()
        rows = []
        for layer in range(2):
            qkv = rand(B, R, Hq + 2 * Hkv, D)
            out = target.attend(layer, qkv, (Hq, Hkv), pos, sec, parents)
            q, k = (x.contiguous() for x in (qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv]))
            sd.rope_apply(q, k, pos, sec)
            rows.append((k, qkv[:, :, Hq + Hkv:]))
            for b in range(B):
                full = [np.swapaxes(np.concatenate([kept[layer][b][j], to64(rows[layer][j][b])]), 0, 1) for j in range(2)]
                o, dev, size = oracle.tree_attention(to64(q[b]), *full, parents[b].tolist(), spread=True)
                bound = 2.0 ** -8 * np.abs(o) + (1.01 * 2.0 ** -8 + 2 * D * 2.0 ** -23 * size) * dev + 2.0 ** -18
                assert (np.abs(to64(out[b]) - o) <= bound).all()
        z = rand(B, R, V)
        tokens = torch.where(torch.rand((B, R), generator=g, device="cuda") < 0.7,
                             z.argmax(-1).gather(1, parents.clamp_min(0).long()), 0).to(torch.int32)
        n_emit, path, out = target.commit(z, tokens, parents)
        for b in range(B):
            p, o, _ = oracle.accept_tree(to64(z[b]), tokens[b].tolist(), parents[b].tolist())
            assert int(n_emit[b]) == len(p) and path[b].tolist()[:len(p)] == p and out[b].tolist()[:len(p)] == o
            lens[b] += len(p)
            for layer in range(2):
                kept[layer][b] = [np.concatenate([kept[layer][b][j], to64(rows[layer][j][b])[p]]) for j in range(2)]
        for cache in target.caches:
            assert cache.len.tolist() == lens
    assert sd.get_device_error() == 0


def test_command(capsys):
    assert paged_tree.main(["--prefix", "300", "--nodes", "17", "--steps", "3", "--scenes", "3"]) == 0
    assert capsys.readouterr().out.count("committed") == 3
