"""Log probabilities at the temperatures whose inverse is the largest that fp32 holds."""
import numpy as np
import pytest
import torch

from paper_2606_31160_gb300 import sd
from tests.helpers import ensure_lib

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [2e-37, 1e-38, 4e-39, 3.2e-39, 3e-39])
@pytest.mark.parametrize("V", [50, 70001])
def test_smallest_temperatures(T, V):
    """Nothing but the largest logits is left: two of them, log 2."""
    ensure_lib()
    rng = np.random.default_rng(V)
    z = torch.from_numpy((np.round(rng.standard_normal((2, V)) * 8) / 8).astype(np.float32)).cuda()
    z[0, 7], z[1, 9], z[1, V - 2] = 20.0, 20.0, 20.0
    lp, h, ids, top = sd.token_logprobs(z, torch.tensor([7, V - 2], dtype=torch.int32, device="cuda"), T, 2)
    want = np.array([0.0, np.log(2)])
    assert np.allclose(h.cpu().numpy(), want, atol=1e-6) and np.allclose(lp.cpu().numpy(), -want, atol=1e-6)
    assert ids[:, 0].tolist() == [7, 9] and ids[1, 1] == V - 2
    assert top[0, 1] < -1e30 and np.allclose(top[1].cpu().numpy(), -np.log(2), atol=1e-6)
    assert sd.get_device_error() == 0
