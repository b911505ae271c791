"""The tree attention's workspace: the size of the largest call is enough for every smaller one."""
import numpy as np
import pytest
import torch

from paper_2606_31160_gb300 import build, sd


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


HEADS = [(32, 8, 128), (28, 4, 64), (16, 4, 128), (8, 8, 64), (7, 1, 128)]


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
def test_the_size_grows_with_scenes_rows_and_capacity(Hq, Hkv, D):
    """(without a device: the size for the largest one that is served)"""
    Bs, Rs, caps = (1, 2, 3, 7, 8, 20, 25, 26, 33, 48, 64, 200), (1, 2, 5, 8, 9, 16, 17, 26, 32, 61, 64, 65, 128, 129, 200, 256), \
        (16, 128, 144, 272, 1024, 4160, 8192, 65536, 131072)
    n = np.array([[[sd.tree_attention_workspace_bytes(B, R, Hq, Hkv, D, cap) for cap in caps] for R in Rs] for B in Bs])
    assert all((np.diff(n, axis=a) >= 0).all() for a in range(3))
    assert (n[..., :2] == 0).all()   # one tile a unit: nothing is ever cut
    assert (n[-1, :, 2:] > 0).all()  # a batch


@pytest.mark.gpu
@pytest.mark.parametrize("Hq,Hkv,D,B,R,keys", [(28, 4, 64, 48, 61, 4000), (32, 8, 128, 26, 26, 4100), (8, 4, 128, 40, 64, 1500)])
def test_one_workspace_for_every_smaller_call(Hq, Hkv, D, B, R, keys):
    """Of the largest call's size, its content anything; the results are those of a call that
    brings none. Some of the calls take a workspace, and say so where it is too short."""
    page = 16
    width = -(-keys // page)
    g = torch.Generator(device="cuda").manual_seed(B)
    pools = [torch.randn((width, Hkv, page, D), generator=g, device="cuda", dtype=torch.bfloat16) for _ in "kv"]
    row = torch.randperm(width, generator=g, device="cuda").to(torch.int32)  # (pages that all scenes share: none is written)
    ws = torch.empty(sd.tree_attention_workspace_bytes(B, R, Hq, Hkv, D, width * page), dtype=torch.uint8, device="cuda")
    none = torch.empty(0, dtype=torch.uint8, device="cuda")
    taken = []
    for b in sorted({1, 2, 8, B // 2, B - 1, B}):
        for cap in (width, width // 2, 9):
            cache = sd.PagedKVCache(*pools, row[:cap].expand(b, cap).contiguous(),
                                    torch.randint(R, min(keys, cap * page) + 1, (b,), generator=g, device="cuda", dtype=torch.int32))
            for r in (1, 8, 17, R):
                q = torch.randn((b, r, Hq, D), generator=g, device="cuda", dtype=torch.bfloat16)
                want = sd.tree_attention(q, cache)
                ws.fill_(255)
                assert torch.equal(sd.tree_attention(q, cache, ws=ws), want)
                try:
                    assert torch.equal(sd.tree_attention(q, cache, ws=none), want)
                    taken.append(False)
                except sd.SDError as e:
                    assert e.status == sd.SD_ERR_WORKSPACE
                    taken.append(True)
    assert any(taken) and not all(taken)
    assert sd.get_device_error() == 0
