"""The attention of drafted trees over a paged cache and the acceptance along a tree,
against the float64 oracle.

The attention's bound, per element o = sum_j w_j v_j: the output's rounding to bf16 (at
most 2^-8 |o|), the weights' (at most 2^-8 of each, numerator and sum alike: 2^-8 sum_j w_j
|v_j - o|, which is at most 2^-8 (sum_j w_j (v_j - o)^2)^(1/2)), and the scores' fp32 sums of D
products (D 2^-23 sum |q k| scale on a score, twice that on a ratio of weights), with 2^-20 of
the largest value for the fp32 sums over keys."""
import numpy as np
import pytest
import torch

import oracle
from helpers import to64
from paper_2606_31160_gb300 import build, sd
from test_gpu_paged import _i32, _randn, make_cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    sd.get_device_error()


def make_tree(rng, n, extend=0.35, forest=False):
    return np.array([-1] + [i - 1 if rng.random() < extend else int(rng.integers(-1 if forest else 0, i)) for i in range(1, n)],
                    dtype=np.int32)


def check_scene(out, q, cache, b, parents, n_new, scale=None):
    n = int(cache.len[b])
    m = int(n_new)
    table = cache.table[b].cpu().numpy()
    k, v = (oracle.gather_pages(to64(getattr(cache, w)), table, n) for w in "kv")
    o, dev, size = oracle.tree_attention(to64(q[b, :m]), k, v, parents[:m], scale, spread=True)
    D = q.shape[-1]
    finite = np.isfinite(o)
    got = to64(out[b, :m])
    assert np.array_equal(np.isfinite(got), finite)
    big = np.abs(v[np.isfinite(v)]).max() if v.size else 0.0
    with np.errstate(invalid="ignore"):
        bound = 2.0 ** -8 * np.abs(o) + (1.01 * 2.0 ** -8 + 2 * D * 2.0 ** -23 * size) * dev + 2.0 ** -20 * big
        bad = finite & ~(np.abs(got - o) <= bound)
    assert not bad.any(), (b, np.argwhere(bad)[:5], np.abs(got - o)[bad][:5], bound[bad][:5])


CASES = [
    # B, R, Hq, Hkv, D, prefix (largest), page, tree, ragged
    (1, 1, 4, 1, 64, 0, 16, False, False),          # a single row that sees itself alone
    (1, 1, 16, 4, 128, 1, 16, False, False),
    (1, 1, 16, 4, 128, 300, 128, False, False),
    (1, 8, 32, 8, 128, 1000, 64, False, False),     # a chain: the causal mask
    (2, 8, 8, 8, 128, 127, 16, True, True),
    (3, 13, 28, 4, 64, 259, 32, True, True),
    (1, 26, 32, 8, 128, 515, 64, True, False),
    (2, 33, 8, 4, 64, 640, 16, True, True),
    (2, 61, 16, 4, 128, 200, 32, True, True),       # 244 packed rows a KV head
    (1, 128, 4, 4, 128, 0, 16, True, False),        # no prefix
    (2, 130, 4, 2, 64, 90, 64, True, True),         # more than 256 packed rows
    (1, 256, 3, 1, 128, 129, 128, True, False),     # three m-blocks, the largest tree
    (5, 3, 7, 1, 128, 60, 16, True, True),          # an odd group
    (9, 4, 10, 2, 64, 300, 32, True, True),
    # many tiles a CTA, for every number of packed rows and both head dims
    (1, 2, 8, 8, 128, 27000, 128, False, False),
    (3, 3, 16, 8, 64, 21000, 64, True, True),
    (2, 12, 32, 8, 128, 11000, 16, True, False),
    (2, 30, 24, 8, 64, 16001, 128, True, True),
    (5, 13, 56, 8, 128, 5003, 64, True, True),
    (3, 61, 32, 8, 128, 6000, 64, True, True),
    (2, 40, 32, 4, 64, 13000, 32, True, False),
]


@pytest.mark.parametrize("B,R,Hq,Hkv,D,prefix,page,tree,ragged", CASES)
def test_attention(B, R, Hq, Hkv, D, prefix, page, tree, ragged):
    g = torch.Generator(device="cuda").manual_seed(R + prefix)
    rng = np.random.default_rng(R + 7 * B)
    n_new = rng.integers(0, R + 1, B) if ragged else np.full(B, R)
    if ragged:
        n_new[-1] = R
    lens = (rng.integers(0, prefix + 1, B) if B > 1 else np.full(B, prefix)) + n_new
    cache = make_cache(g, lens, prefix + R, Hkv, D, page)
    cache.k[:, :, :, 3] *= 4  # scores well away from one another
    parents = np.stack([make_tree(rng, R, forest=True) for _ in range(B)]) if tree else np.tile(np.arange(R) - 1, (B, 1))
    for b in range(B):  # rows past the last are anything
        t, n = cache.table[b], int(lens[b])
        for at in range(n, t.numel() * page):
            cache.k[t[at // page], :, at % page] = float("nan")
            cache.v[t[at // page], :, at % page] = float("inf")
    q = _randn(g, B, R, Hq, D)
    bad = parents.copy()
    for b in range(B):
        bad[b, n_new[b]:] = 1 << 20  # as are the other rows' parents
    out = torch.full((B, R, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    got = sd.tree_attention(q, cache, parents=_i32(bad) if tree else None, n_new=_i32(n_new) if ragged else None, out=out)
    assert got is out and sd.get_device_error() == 0
    for b in range(B):
        check_scene(out, q, cache, b, parents[b], n_new[b])
        assert (out[b, n_new[b]:] == 7.0).all()


def test_attention_of_a_chain_is_the_verify_attention():
    """The same rows, keys and mask as sd.verify_attention: within both kernels' bounds."""
    g = torch.Generator(device="cuda").manual_seed(0)
    B, R, Hq, Hkv, D, L = 2, 8, 32, 8, 128, 700
    cache = make_cache(g, [L, L - 99], L, Hkv, D, 64)
    kv = sd.KVCache(*(x[cache.table.long()].transpose(1, 2).reshape(B, Hkv, -1, D).contiguous() for x in (cache.k, cache.v)),
                    cache.len.clone())
    q = _randn(g, B, R, Hq, D)
    a, b = sd.tree_attention(q, cache).float(), sd.verify_attention(q, kv).float()
    chain = sd.tree_attention(q, cache, parents=_i32(np.tile(np.arange(R) - 1, (B, 1))))
    assert torch.equal(chain.float(), a) and (a - b).abs().max() <= 2e-2
    assert sd.get_device_error() == 0


@pytest.mark.parametrize("Hq,Hkv,R", [(4, 1, 6), (8, 1, 8), (8, 1, 14), (8, 1, 28)])
@pytest.mark.parametrize("D", [64, 128])
def test_masked_infinities_and_nan(Hq, Hkv, R, D):
    """A row that does not see a key does not see what is no number in it."""
    g = torch.Generator(device="cuda").manual_seed(R)
    rng = np.random.default_rng(R)
    prefix = 130
    cache = make_cache(g, [prefix + R], prefix + R, Hkv, D, 16)
    parents = make_tree(rng, R)
    t = cache.table[0]
    for row, key, value in ((R - 1, float("nan"), 1.0), (R - 2, None, float("inf")), (R // 2, 1.0, float("nan")),
                            (R // 2 + 1, None, -float("inf"))):
        at = prefix + row
        if key is not None:
            cache.k[t[at // 16], :, at % 16, 5] = key
        cache.v[t[at // 16], :, at % 16, 7] = value
    q = _randn(g, 1, R, Hq, D)
    out = sd.tree_attention(q, cache, parents=_i32(parents[None]))
    assert sd.get_device_error() == 0
    k, v = (oracle.gather_pages(to64(getattr(cache, w)), t.cpu().numpy(), prefix + R) for w in "kv")
    want, got = oracle.tree_attention(to64(q[0]), k, v, parents), to64(out[0])
    assert np.array_equal(np.isfinite(want), np.isfinite(got)) and np.isfinite(want).any() and not np.isfinite(want).all()
    check_scene(out, q, cache, 0, parents, R)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("R", [1, 14, 30, 60])
@pytest.mark.parametrize("at", [0, 200])
def test_values_of_the_prefix_that_are_no_numbers(R, D, at):
    """They reach every row of their KV head, in their column alone; a key's, all columns."""
    g = torch.Generator(device="cuda").manual_seed(R)
    prefix, parents = 300, make_tree(np.random.default_rng(R), R)
    cache = make_cache(g, [prefix + R], prefix + R, 3, D, 32)
    t = cache.table[0]
    cache.v[t[at // 32], 0, at % 32, 7] = float("inf")
    cache.v[t[at // 32], 1, at % 32, 9] = float("nan")
    cache.k[t[at // 32], 2, at % 32, 5] = float("nan")
    q = _randn(g, 1, R, 12, D)
    out = sd.tree_attention(q, cache, parents=_i32(parents[None]))
    assert sd.get_device_error() == 0
    want = torch.ones((R, 12, D), dtype=torch.bool, device="cuda")
    want[:, :4, 7] = want[:, 4:8, 9] = want[:, 8:] = False
    assert torch.equal(out[0].isfinite(), want)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("R", [1, 9, 40])
def test_scores_far_from_zero_and_rising(R, D):
    """Keys whose scores rise along the cache, jump late, or lie far below 0; -inf scores."""
    g = torch.Generator(device="cuda").manual_seed(5)
    Hq, Hkv, L = 4, 2, 900
    q = _randn(g, 1, R, Hq, D)
    q[..., 0] = 4.0
    up = torch.arange(L, device="cuda") / L
    for shape in (up * 200, -up * 200, torch.where(up > 0.7, 250.0, -250.0), torch.full_like(up, -3e4),
                  torch.where(up < 0.5, -float("inf"), 0.0)):
        cache = make_cache(g, [L], L, Hkv, D, 32)
        at = torch.arange(L, device="cuda")
        cache.k[cache.table[0, at // 32].long(), :, at % 32, 0] = (shape / 4)[:, None].to(torch.bfloat16).expand(-1, Hkv)
        out = sd.tree_attention(q, cache)
        assert sd.get_device_error() == 0
        check_scene(out, q, cache, 0, np.arange(R) - 1, R)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("R", [1, 24, 60, 110])
def test_references_that_move_in_a_run(R, D):
    """Scores that rise over many tiles of a CTA, by little and by much, in every row tile: the
    references move and what was summed with them."""
    g = torch.Generator(device="cuda").manual_seed(R)
    Hq, Hkv, L = 8, 4, 20000
    q = _randn(g, 1, R, Hq, D)
    q[..., 0] = 4.0
    up = torch.arange(L, device="cuda") / L
    for shape in (up * 120, (up * 8).floor() * 90, torch.where((up > 0.6) & (up < 0.6001), 300.0, 0.0)):
        cache = make_cache(g, [L], L, Hkv, D, 64)
        at = torch.arange(L, device="cuda")
        cache.k[cache.table[0, at // 64].long(), :, at % 64, 0] = (shape / 4 * (D / 64) ** 0.5)[:, None].to(torch.bfloat16).expand(-1, Hkv)
        out = sd.tree_attention(q, cache)
        assert sd.get_device_error() == 0
        check_scene(out, q, cache, 0, np.arange(R) - 1, R)


@pytest.mark.parametrize("B,R,Hq,Hkv,D,L", [(100, 5, 4, 2, 64, 3000), (80, 15, 8, 2, 64, 4000), (80, 30, 8, 2, 128, 3000),
                                              (40, 33, 16, 4, 128, 5000), (42, 70, 8, 4, 64, 3500)])
def test_attention_of_many_scenes(B, R, Hq, Hkv, D, L):
    """More than 32 scenes, in even shares (the way that takes a workspace), some with nothing
    new and some not valid; the workspace of any content, the results the same every time."""
    assert sd.tree_attention_workspace_bytes(B, R, Hq, Hkv, D, -(-(L + R) // 64) * 64) > 0
    g = torch.Generator(device="cuda").manual_seed(B)
    rng = np.random.default_rng(B)
    n_new = rng.integers(0, R + 1, B)
    n_new[0], n_new[-1] = R, R
    lens = rng.integers(0, L + 1, B) + n_new
    cache = make_cache(g, lens, L + R, Hkv, D, 64)
    parents = np.stack([make_tree(rng, R, forest=True) for _ in range(B)])
    bad_len, bad_tree, bad_page = 7, B // 2, B - 2
    n_new[bad_tree] = n_new[bad_page] = R
    lens[bad_tree], lens[bad_page] = L + R, L + R
    cache.len.copy_(_i32(lens))
    cache.len[bad_len] = -1
    parents[bad_tree, R // 2] = R
    cache.table[bad_page, 3] = -1
    q = _randn(g, B, R, Hq, D)
    ws = torch.full((sd.tree_attention_workspace_bytes(B, R, Hq, Hkv, D, cache.shape[2]),), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.full((B, R, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    sd.tree_attention(q, cache, parents=_i32(parents), n_new=_i32(n_new), out=out, ws=ws)
    assert sd.get_device_error() == sd.SD_DEVERR_LENGTH | sd.SD_DEVERR_TREE | sd.SD_DEVERR_PAGE
    for b in range(B):
        if b in (bad_len, bad_tree):
            assert (out[b] == 7.0).all()
        elif b == bad_page:
            assert out[b].isnan().all()
        else:
            check_scene(out, q, cache, b, parents[b], n_new[b])
            assert (out[b, n_new[b]:] == 7.0).all()
    again = sd.tree_attention(q, cache, parents=_i32(parents), n_new=_i32(n_new), out=torch.full_like(out, 7.0))
    assert torch.equal(again.view(torch.int16), out.view(torch.int16))
    sd.get_device_error()


def test_two_graphs_and_a_workspace_of_ones_own():
    """Two captured graphs that share a workspace, replayed in turn, each the same as its call;
    a workspace that is too short is refused."""
    g = torch.Generator(device="cuda").manual_seed(3)
    B, R, Hq, Hkv, D, L = 40, 6, 8, 4, 128, 1500
    need = sd.tree_attention_workspace_bytes(B, R, Hq, Hkv, D, -(-L // 32) * 32)
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    sides = []
    for _ in range(2):
        cache = make_cache(g, [L - 7 * b for b in range(B)], L, Hkv, D, 32)
        sides.append((_randn(g, B, R, Hq, D), cache, torch.zeros((B, R, Hq, D), dtype=torch.bfloat16, device="cuda")))
    want = [sd.tree_attention(q, cache) for q, cache, _ in sides]
    torch.cuda.synchronize()
    graphs = []
    for q, cache, out in sides:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            sd.tree_attention(q, cache, out=out, ws=ws)
        graphs.append(graph)
    for _ in range(3):
        for i, graph in enumerate(graphs):
            graph.replay()
            assert torch.equal(sides[i][2], want[i])
    assert sd.get_device_error() == 0
    with pytest.raises(sd.SDError) as e:
        sd.tree_attention(sides[0][0], sides[0][1], ws=ws[:need - 16])
    assert e.value.status == 3


def test_a_long_tail_beside_one_key():
    """One key that holds most of a row over thousands that share the rest."""
    g = torch.Generator(device="cuda").manual_seed(6)
    Hq, Hkv, L, D = 4, 1, 5000, 128
    for at in (0, 2600, L - 1):
        for share in (0.5, 0.99):
            cache = make_cache(g, [L], L, Hkv, D, 64)
            cache.k.zero_()
            cache.v[cache.v.isnan()] = 0
            cache.v.fill_(1.0)
            cache.k[cache.table[0, at // 64], :, at % 64, 0] = 1.0
            cache.v[cache.table[0, at // 64], :, at % 64] = -1.0
            q = torch.zeros((1, 1, Hq, D), dtype=torch.bfloat16, device="cuda")
            q[..., 0] = float(np.log(share / (1 - share) * (L - 1)) * D ** 0.5)
            out = sd.tree_attention(q, cache)
            check_scene(out, q, cache, 0, np.array([-1]), 1)


def test_attention_scale_strides_and_shared_pages():
    g = torch.Generator(device="cuda").manual_seed(7)
    B, R, Hq, Hkv, D = 3, 11, 8, 2, 64
    rng = np.random.default_rng(7)
    cache = make_cache(g, [150 + R] * B, 150 + R, Hkv, D, 16)
    cache.table[1, :8], cache.table[2, :9] = cache.table[0, :8], cache.table[0, :9]  # a prefix that scenes share
    qkv = _randn(g, B, R, Hq + 2 * Hkv, D)
    q = qkv[:, :, :Hq]
    parents = np.stack([make_tree(rng, R) for _ in range(B)])
    for scale in (0.0, 0.03, 1.0):
        out = sd.tree_attention(q, cache, parents=_i32(parents), scale=scale)
        for b in range(B):
            check_scene(out, q, cache, b, parents[b], R, scale or None)
    out = sd.tree_attention(q.contiguous(), cache, parents=_i32(parents), scale=1.0)
    assert torch.equal(out, sd.tree_attention(q, cache, parents=_i32(parents), scale=1.0))
    with pytest.raises(ValueError):
        sd.tree_attention(qkv.transpose(0, 1), cache)
    with pytest.raises(ValueError):
        sd.tree_attention(qkv[..., ::2], cache)
    assert sd.get_device_error() == 0


def test_attention_errors():
    g = torch.Generator(device="cuda").manual_seed(8)
    B, R, Hq, Hkv, D, page = 3, 7, 4, 2, 64, 16
    q = _randn(g, B, R, Hq, D)
    parents = np.tile(np.array([-1, 0, 0, 1, 1, 2, 4]), (B, 1))

    def check(bit, lens=(50, 300, 20), parents=parents, n_new=(7, 7, 7), entry=None, nan=False):
        cache = make_cache(g, [60, 300, 30], 400, Hkv, D, page)
        cache.len.copy_(_i32(lens))
        if entry is not None:
            cache.table[1, entry[0]] = entry[1]
        out = torch.full((B, R, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
        sd.tree_attention(q, cache, parents=_i32(parents), n_new=_i32(n_new), out=out)
        assert sd.get_device_error() == bit
        assert out[1].isnan().all() if nan else (out[1] == 7.0).all()
        for b in (0, 2):
            check_scene(out, q, cache, b, parents[b], n_new[b])

    check(0, n_new=(7, 0, 3))
    check(sd.SD_DEVERR_LENGTH, lens=(50, 6, 20))
    check(sd.SD_DEVERR_LENGTH, lens=(50, 401, 20))
    check(sd.SD_DEVERR_LENGTH, n_new=(7, 8, 7))
    check(sd.SD_DEVERR_LENGTH, n_new=(7, -1, 7))
    check(sd.SD_DEVERR_LENGTH, lens=(50, -5, 20), n_new=(7, 0, 7))
    for i, p in ((0, 0), (3, 3), (3, 5), (2, -2), (6, 1 << 30), (6, -(1 << 31))):
        other = parents.copy()
        other[1, i] = p
        check(sd.SD_DEVERR_TREE, parents=other)
    for at, entry in ((0, -1), (7, 1 << 30), (18, -5), (18, 200)):
        check(sd.SD_DEVERR_PAGE, entry=(at, entry), nan=True)
    check(0, lens=(50, 288, 20), entry=(18, -1), n_new=(7, 0, 7))  # (a page behind the last row)


# ------------------------------------------------------------------ acceptance

def accept_case(rng, B, R, V, dtype, n_new, forest=False):
    z = torch.from_numpy(rng.integers(-40, 40, (B, R, V)).astype(np.float32) / 8).to(dtype)
    parents = np.stack([make_tree(rng, R, forest=forest) for _ in range(B)])
    star = to64(z).argmax(-1)
    tokens = rng.integers(0, V, (B, R))
    agree = rng.random((B, R)) < 0.6
    up = np.take_along_axis(star, np.maximum(parents, 0), 1)
    tokens = np.where(agree, up, tokens)
    tokens[:, 0] = 1 << 30  # row 0's is not read
    for b in range(B):
        tokens[b, n_new[b]:], parents[b, n_new[b]:] = -7, 1 << 20
    return z, tokens.astype(np.int32), parents


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,R,V,ragged", [(1, 1, 1, False), (1, 1, 5000, False), (2, 8, 33, False), (5, 26, 4097, True),
                                          (3, 61, 20003, True), (2, 256, 1001, True), (40, 3, 12345, True)])
def test_accept(B, R, V, ragged, dtype):
    rng = np.random.default_rng(B * 100 + R)
    n_new = rng.integers(0, R + 1, B) if ragged else np.full(B, R)
    z, tokens, parents = accept_case(rng, B, R, V, dtype, n_new)
    ws = sd.workspace(sd.accept_tree_workspace_bytes(B, R, V))
    argmax = torch.full((B, R), 77, dtype=torch.int32, device="cuda")
    zc = z.cuda()
    for _ in range(2):  # the workspace is left ready
        n_emit, path, out, best = sd.accept_tree(zc, _i32(tokens), _i32(parents), n_new=_i32(n_new) if ragged else None, ws=ws,
                                                 argmax=argmax)
        assert sd.get_device_error() == 0 and best is argmax
        for b in range(B):
            n = int(n_new[b])
            p, o, star = oracle.accept_tree(to64(z[b, :n]), tokens[b, :n], parents[b, :n])
            assert int(n_emit[b]) == len(p)
            assert path[b].tolist() == p + [-1] * (R - len(p)) and out[b].tolist() == o + [-1] * (R - len(p))
            assert argmax[b].tolist() == star + [77] * (R - n)
    assert (ws == 0).all()


def test_accept_of_a_chain_is_accept_greedy():
    rng = np.random.default_rng(0)
    z = torch.from_numpy(rng.integers(0, 30, (6, 9, 3001)).astype(np.float32)).cuda()
    draft = torch.where(torch.rand((6, 8), device="cuda") < 0.7, z[:, :8].argmax(-1), 5).to(torch.int32)
    tokens = torch.cat([torch.zeros((6, 1), dtype=torch.int32, device="cuda"), draft], 1)
    a, b = sd.accept_greedy(z, draft), sd.accept_tree(z, tokens)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[2]) and torch.equal(a[2], b[3])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_accept_rows_of_any_alignment(dtype):
    rng = np.random.default_rng(1)
    for V, pad, off in ((1000, 0, 0), (1001, 6, 3), (37, 1, 1), (4099, 13, 5)):
        B, R = 3, 5
        z, tokens, parents = accept_case(rng, B, R, V, dtype, np.full(B, R))
        buf = torch.full((B * R * (V + pad) + off,), 1e4, device="cuda").to(dtype)
        rows = buf[off:].view(B, R, V + pad)[..., :V]
        rows.copy_(z)
        got = sd.accept_tree(rows, _i32(tokens), _i32(parents))
        for b in range(B):
            p, o, star = oracle.accept_tree(to64(z[b]), tokens[b], parents[b])
            assert got[1][b].tolist() == p + [-1] * (R - len(p)) and got[3][b].tolist() == star
        assert sd.get_device_error() == 0


def test_accept_ties_signed_zero_and_infinities():
    V = 70000
    z = torch.full((1, 4, V), -float("inf"), device="cuda")
    z[0, 0, [40000, 69999]] = 3.0
    z[0, 1, 500], z[0, 1, 60000] = -0.0, 0.0
    z[0, 3, 65000] = float("inf")
    for zz in (z, z.to(torch.bfloat16)):
        got = sd.accept_tree(zz, _i32([[0, 40000, 500, 0]]))
        assert got[3].tolist() == [[40000, 500, 0, 65000]] and got[1].tolist() == [[0, 1, 2, 3]]
    # several children with the right token: the lowest
    got = sd.accept_tree(z, _i32([[0, 1, 40000, 40000]]), _i32([[-1, 0, 0, 0]]))
    assert got[1].tolist() == [[0, 2, -1, -1]] and got[2].tolist() == [[40000, 0, -1, -1]]


def test_accept_errors():
    rng = np.random.default_rng(2)
    B, R, V = 3, 6, 500
    z, tokens, parents = accept_case(rng, B, R, V, torch.float32, np.full(B, R))
    zc = z.cuda()
    ws = sd.workspace(sd.accept_tree_workspace_bytes(B, R, V))

    def run(bit, tokens=tokens, parents=parents, n_new=(R, R, R), unwritten=True):
        outs = [torch.full(s, 77, dtype=torch.int32, device="cuda") for s in ((B,), (B, R), (B, R), (B, R))]
        sd.accept_tree(zc, _i32(tokens), _i32(parents), n_new=_i32(n_new), ws=ws, n_emit=outs[0], path=outs[1], out=outs[2],
                       argmax=outs[3])
        assert sd.get_device_error() == bit and (ws == 0).all()
        if unwritten:
            assert all((x[1] == 77).all() for x in outs)
        for b in (0, 2):
            assert outs[1][b].tolist()[:int(outs[0][b])] == oracle.accept_tree(to64(z[b]), tokens[b], parents[b])[0]
        return outs

    for i, p in ((0, 0), (2, 2), (5, -2), (5, 1 << 30)):
        other = parents.copy()
        other[1, i] = p
        run(sd.SD_DEVERR_TREE, parents=other)
    run(sd.SD_DEVERR_LENGTH, n_new=(R, R + 1, R))
    run(sd.SD_DEVERR_LENGTH, n_new=(R, -1, R))
    outs = run(0, n_new=(R, 0, R), unwritten=False)
    assert outs[0][1] == 0 and outs[1][1].tolist() == [-1] * R and outs[2][1].tolist() == [-1] * R and (outs[3][1] == 77).all()
    other = tokens.copy()
    other[1, 1:] = [V, -1, 1 << 30, V, -5]
    outs = run(sd.SD_DEVERR_TOKEN_RANGE, tokens=other, unwritten=False)
    assert outs[1][1].tolist() == [0] + [-1] * (R - 1)


# ------------------------------------------------------------------ together

@pytest.mark.parametrize("graph", [False, True])
def test_a_step_over_pages(graph):
    """Append, attention, acceptance, commit, as a serving loop runs them, twice, against the
    same steps by hand; also captured in a graph and replayed."""
    g = torch.Generator(device="cuda").manual_seed(11)
    rng = np.random.default_rng(11)
    B, R, Hq, Hkv, D, V, layers, sec = 3, 12, 8, 2, 128, 997, 2, (16, 24, 24)
    caches = [make_cache(g, [40, 200, 7], 300, Hkv, D, 16) for _ in range(layers)]
    group = sd.PagedKVCacheGroup(caches)
    bufs = dict(qkv=_randn(g, layers, B, R, Hq + 2 * Hkv, D), pos=_i32(np.zeros((B, R, 3))), parents=_i32(np.zeros((B, R))),
                tokens=_i32(np.zeros((B, R))), n_new=_i32(np.zeros(B)), z=torch.zeros((B, R, V), device="cuda"))
    ws = sd.workspace(sd.accept_tree_workspace_bytes(B, R, V))
    q_rot = torch.zeros((layers, B, R, Hq, D), dtype=torch.bfloat16, device="cuda")
    out = torch.zeros_like(q_rot)
    res = [torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((B,), (B, R), (B, R), (B, R))]

    def step():
        for i, cache in enumerate(caches):
            q, k, v = bufs["qkv"][i].split([Hq, Hkv, Hkv], dim=2)
            sd.paged_append(cache, k, v, q=q, pos=bufs["pos"], sections=sec, n_new=bufs["n_new"], q_out=q_rot[i])
            sd.tree_attention(q_rot[i], cache, parents=bufs["parents"], n_new=bufs["n_new"], out=out[i])
        sd.accept_tree(bufs["z"], bufs["tokens"], bufs["parents"], n_new=bufs["n_new"], ws=ws, n_emit=res[0], path=res[1],
                       out=res[2], argmax=res[3])
        sd.paged_commit(group, res[1], res[0], n_new=bufs["n_new"])

    replay = step
    if graph:
        step()  # (n_new 0: nothing moves)
        torch.cuda.synchronize()
        graph_ = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph_):
            step()
        replay = graph_.replay
    lens = [40, 200, 7]
    rows = [[[np.swapaxes(oracle.gather_pages(to64(getattr(c, w)), c.table[b].cpu().numpy(), lens[b]), 0, 1) for w in "kv"]
             for b in range(B)] for c in caches]
    for it in range(2):
        n_new = np.array([R, 5, 1]) if it == 0 else np.array([0, R, 9])
        z, tokens, parents = accept_case(rng, B, R, V, torch.float32, n_new)
        depth = np.zeros((B, R), dtype=np.int64)
        for b in range(B):
            for i in range(1, n_new[b]):
                depth[b, i] = depth[b, parents[b, i]] + 1
        pos = np.repeat((np.array(lens)[:, None] + depth)[..., None], 3, -1)
        for name, x in (("pos", _i32(pos)), ("parents", _i32(parents)), ("tokens", _i32(tokens)), ("n_new", _i32(n_new)), ("z", z)):
            bufs[name].copy_(x)
        bufs["qkv"].copy_(_randn(g, *bufs["qkv"].shape))
        replay()
        assert sd.get_device_error() == 0
        for b in range(B):
            n = n_new[b]
            p, o, _ = oracle.accept_tree(to64(z[b, :n]), tokens[b, :n], parents[b, :n])
            assert int(res[0][b]) == len(p) and res[1][b].tolist()[:len(p)] == p and res[2][b].tolist()[:len(p)] == o
            for i, c in enumerate(caches):
                q, k, v = bufs["qkv"][i, b, :n].split([Hq, Hkv, Hkv], dim=1)
                q1, k1 = q.contiguous()[None], k.contiguous()[None]
                if n:
                    sd.rope_apply(q1, k1, _i32(pos[b:b + 1, :n]), sec)
                    full = [np.concatenate([rows[i][b][j], to64(x)]) for j, x in enumerate((k1[0], v))]
                    want, dev, size = oracle.tree_attention(to64(q1[0]), *(np.swapaxes(x, 0, 1) for x in full), parents[b, :n], spread=True)
                    bound = 2.0 ** -8 * np.abs(want) + (1.01 * 2.0 ** -8 + 2 * D * 2.0 ** -23 * size) * dev + 2.0 ** -18
                    assert (np.abs(to64(out[i, b, :n]) - want) <= bound).all()
                else:
                    full = rows[i][b]
                rows[i][b] = [np.array(oracle.commit_rows(list(x), n, p)).reshape(-1, Hkv, D) for x in full]
                assert int(c.len[b]) == lens[b] + len(p)
                for j, w in enumerate("kv"):
                    got = np.swapaxes(oracle.gather_pages(to64(getattr(c, w)), c.table[b].cpu().numpy(), lens[b] + len(p)), 0, 1)
                    assert np.array_equal(got, rows[i][b][j])
            lens[b] += len(p)


def test_another_stream():
    g = torch.Generator(device="cuda").manual_seed(12)
    cache = make_cache(g, [500], 512, 4, 128, 32)
    q = _randn(g, 1, 6, 16, 128)
    want = sd.tree_attention(q, cache)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = sd.tree_attention(q, cache)
        z = torch.randn((1, 6, 999), device="cuda")
        a = sd.accept_tree(z, torch.zeros((1, 6), dtype=torch.int32, device="cuda"))
    s.synchronize()
    assert torch.equal(got, want) and a[3][0].tolist() == z[0].argmax(-1).tolist()
    assert sd.get_device_error() == 0
