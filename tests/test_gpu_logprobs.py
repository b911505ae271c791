"""GPU parity of token_logprobs against the float64 oracle."""
import numpy as np
import pytest
import torch

import oracle
from paper_2606_31160_gb300 import sd
from tests.helpers import ensure_lib, to64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_lib()
    sd.get_device_error()


def _check(z, tokens, T=1.0, n=0):
    lead = tokens.shape
    lp, h, ids, top = sd.token_logprobs(z, tokens, T, n)
    assert tuple(lp.shape) == lead and tuple(ids.shape) == lead + (n,)
    V = z.shape[-1]
    z64 = to64(z).reshape(-1, V)
    rl, rh, ri, rt = oracle.token_logprobs(z64, tokens.cpu().numpy().reshape(-1), T, n)
    # fp32: x = (z - max) / T is off by two roundings of it, ln S by a few 2^-23 of a sum
    # of positive terms; the entropy adds S and W of relative errors as small
    near = lambda a, r: np.all((np.abs(a - r) <= 4e-6 + 2.0 ** -21 * np.abs(r)) | (a == r))  # noqa: E731
    assert near(to64(lp).reshape(-1), rl)
    assert near(to64(h).reshape(-1), rh)
    assert np.array_equal(ids.cpu().numpy().reshape(len(z64), n), ri)
    assert near(to64(top).reshape(len(z64), n), rt)
    assert sd.get_device_error() == 0


def _tokens(rng, lead, V):
    t = rng.integers(0, V, lead)
    t[..., -1:] = np.where(rng.random(t[..., -1:].shape) < 0.5, -1, t[..., -1:])
    return torch.from_numpy(t.astype(np.int32)).cuda()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lead,V,n,T", [
    ((1, 1), 1, 1, 1.0), ((2,), 7, 7, 0.5), ((3, 2), 31, 5, 1.0), ((1, 5), 33, 32, 2.0), ((2, 3), 1000, 0, 0.6),
    ((1, 8), 50257, 20, 1.0), ((4, 9), 4096, 32, 0.7), ((1, 2), 151936, 5, 1.3), ((2, 17), 32000, 1, 1.0),
    ((40, 8), 2049, 3, 1.0), ((3,), 65537, 20, 0.6), ((1,), 300001, 32, 1.0),
])
def test_parity(dtype, lead, V, n, T):
    rng = np.random.default_rng(V + n)
    z = torch.from_numpy((rng.standard_normal(lead + (V,)) * 3).astype(np.float32)).to(dtype).cuda()
    _check(z, _tokens(rng, lead, V), T, n)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_orders_and_ties(dtype):
    """Rising, falling, all equal, few values, one far above the rest, -0 beside +0."""
    V = 5000
    rng = np.random.default_rng(1)
    x = np.linspace(-9, 9, V)
    z = np.stack([x, x[::-1], np.zeros(V), rng.integers(0, 3, V), np.where(np.arange(V) == 4321, 80.0, x),
                  np.where(np.arange(V) % 2 == 0, -0.0, 0.0), -1e30 * np.ones(V), np.where(np.arange(V) < 2500, -200.0, 200.0)])
    z = torch.from_numpy(z.astype(np.float32)).to(dtype).cuda()
    _check(z, _tokens(rng, (8,), V), 1.0, 32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_masked_vocabulary(dtype):
    rng = np.random.default_rng(2)
    z = rng.standard_normal((4, 3000)).astype(np.float32)
    z[0, 5:] = -np.inf       # five tokens left, ten alternatives asked
    z[1, :2990] = -np.inf
    z[2, ::2] = -np.inf
    z[3, 1:] = -np.inf       # one: its entropy is 0
    tokens = torch.tensor([7, 2999, 0, 0], dtype=torch.int32, device="cuda")
    _check(torch.from_numpy(z).to(dtype).cuda(), tokens, 0.8, 10)


def test_rows_without_a_distribution():
    z = torch.zeros((4, 100), device="cuda")
    z[0] = -float("inf")
    z[1, 50] = float("inf")
    z[2, 50] = float("nan")
    lp, h, ids, top = sd.token_logprobs(z, torch.tensor([3, 50, 3, 3], dtype=torch.int32, device="cuda"), 1.0, 4)
    assert lp[:3].isnan().all() and h[:3].isnan().all() and top[:3].isnan().all() and not lp[3].isnan()
    assert ids[0].tolist() == [0, 1, 2, 3] and ids[1, 0] == 50 and ((ids >= 0) & (ids < 100)).all()
    assert sd.get_device_error() == 0


def test_tokens_out_of_range():
    z = torch.randn((4, 100), device="cuda")
    lp = sd.token_logprobs(z, torch.tensor([-1, 100, -2, 99], dtype=torch.int32, device="cuda"))[0]
    assert sd.get_device_error() == sd.SD_DEVERR_TOKEN_RANGE
    assert lp[0] == 0 and lp[1].isnan() and lp[2].isnan() and torch.isfinite(lp[3])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pad", [1, 3, 8, 64])
def test_padded_rows(dtype, pad):
    """Rows of a padded vocabulary: every alignment of a row's start; the padding is not read."""
    rng = np.random.default_rng(pad)
    full = torch.full((2, 5, 1001 + pad), float("nan"), dtype=dtype, device="cuda")
    full[..., :1001] = torch.from_numpy(rng.standard_normal((2, 5, 1001)).astype(np.float32)).to(dtype).cuda()
    _check(full[..., :1001], _tokens(rng, (2, 5), 1001), 1.0, 9)
    with pytest.raises(ValueError):
        sd.token_logprobs(full[:, ::2, :1001].transpose(0, 1), torch.zeros((3, 2), dtype=torch.int32, device="cuda"))


def test_deterministic():
    z = torch.randn((16, 60000), device="cuda").to(torch.bfloat16)
    t = torch.randint(0, 60000, (16,), device="cuda").to(torch.int32)
    first = sd.token_logprobs(z, t, 0.9, 20)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(sd.token_logprobs(z, t, 0.9, 20), first))
