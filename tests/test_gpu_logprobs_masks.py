"""Log probabilities and entropies of rows whose masked tokens hold large finite numbers
(the type's lowest value, -1e38) in place of -inf."""
import numpy as np
import pytest
import torch

import oracle
from paper_2606_31160_gb300 import sd
from tests.helpers import ensure_lib, to64

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float32]


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_lib()
    sd.get_device_error()


def _check(z, tokens, T, n):
    """Against the oracle, its numbers as fp32 holds them (what passes its range is -inf)."""
    lp, h, ids, top = sd.token_logprobs(z, tokens, T, n)
    rl, rh, ri, rt = oracle.token_logprobs(to64(z), tokens.cpu().numpy(), T, n)
    with np.errstate(over="ignore"):
        rl, rt = rl.astype(np.float32).astype(np.float64), rt.astype(np.float32).astype(np.float64)
    # fp32: x = (z - max) / T is off by two roundings of it, ln S by a few 2^-23 of a sum
    # of positive terms; the entropy adds S and W of relative errors as small
    def near(a, r):
        return np.all((a == r) | (np.abs(a - np.where(a == r, a, r)) <= 4e-6 + 2.0 ** -21 * np.abs(np.where(a == r, 0.0, r))))
    assert near(to64(h), rh), (to64(h), rh)
    assert near(to64(lp), rl)
    assert np.array_equal(ids.cpu().numpy(), ri)
    assert near(to64(top), rt)
    assert sd.get_device_error() == 0


def _lowest(dtype):
    return torch.finfo(dtype).min


def _rows(dtype, V, low, seed):
    """Rows of ordinary logits with `low` in runs of them: interleaved, whole warps' chunks,
    the first and the last half, all but a few, all but one, all but the last."""
    g = torch.Generator().manual_seed(seed)
    z = torch.randn((8, V), generator=g) * 3
    at = torch.arange(V)
    z[0, at % 2 == 0] = low
    z[1, (at // 512) % 3 != 0] = low
    z[2, : V // 2] = low
    z[3, V // 2:] = low
    z[4, 40:] = low
    z[5] = torch.where(at == V // 3, z[5], torch.tensor(low))
    z[6, :-1] = low
    z[7, torch.rand(V, generator=g) < 0.3] = low
    return z.to(dtype).cuda()


# (several CTAs a row: whole segments of masked logits)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [40, 1000, 50257, 151936])
@pytest.mark.parametrize("T", [0.3, 1.0, 2.0])
@pytest.mark.parametrize("low", ["lowest", -1e38, -1e37, -1e30])
def test_finite_masks(dtype, V, T, low):
    low = _lowest(dtype) if low == "lowest" else low
    z = _rows(dtype, V, low, V)
    tokens = z.float().argmax(-1).to(torch.int32)
    tokens[7] = -1
    _check(z, tokens, T, min(20, V))


@pytest.mark.parametrize("dtype", DTYPES)
def test_uniform_over_what_is_left(dtype):
    """2^k tokens of one logit, the rest masked: entropy k ln 2."""
    V = 30000
    for k in (0, 1, 5, 11):
        z = torch.full((2, V), _lowest(dtype), dtype=dtype, device="cuda")
        z[0, 17:17 + 2 ** k] = 2.5
        z[1, -2 ** k:] = -60.0
        lp, h, _, _ = sd.token_logprobs(z, torch.tensor([17, V - 1], dtype=torch.int32, device="cuda"), 0.7)
        # fp32: a few roundings of k ln 2
        assert np.allclose(h.cpu().numpy(), k * np.log(2), rtol=2.0 ** -21, atol=1e-6)
        assert np.allclose(lp.cpu().numpy(), -k * np.log(2), rtol=2.0 ** -21, atol=1e-6)


def test_both_ends_of_the_type():
    """The lowest and the highest number in one row; all lowest: uniform."""
    V = 5000
    low = _lowest(torch.float32)
    z = torch.full((2, V), low, device="cuda")
    z[0, 4321] = -low
    z[0, 7] = 0.0
    lp, h, ids, _ = sd.token_logprobs(z, torch.tensor([4321, 9], dtype=torch.int32, device="cuda"), 1.0, 2)
    assert lp[0] == 0 and h[0] == 0 and ids[0].tolist() == [4321, 7]
    assert np.allclose([lp[1].item(), h[1].item()], [-np.log(V), np.log(V)], rtol=2.0 ** -21)
    assert sd.get_device_error() == 0
