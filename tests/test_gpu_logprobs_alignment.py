"""Log probabilities of logits that begin anywhere: rows of an odd vocabulary sliced from a
batch, any element of a 32-byte line."""
import numpy as np
import pytest
import torch

from paper_2606_31160_gb300 import sd
from tests.helpers import ensure_lib
from tests.test_gpu_logprobs import _check, _tokens

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_lib()
    sd.get_device_error()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_sliced_from_a_batch(dtype):
    rng = np.random.default_rng(0)
    z = torch.from_numpy(rng.standard_normal((4, 3, 5001)).astype(np.float32)).to(dtype).cuda()
    for first in (1, 2, 3):
        part = z[first:]
        assert part.is_contiguous()
        _check(part, _tokens(rng, tuple(part.shape[:-1]), 5001), 0.9, 7)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [3, 40, 1000])
def test_every_element_of_a_line(dtype, V):
    rng = np.random.default_rng(V)
    flat = torch.from_numpy(rng.standard_normal(5 * V + 40).astype(np.float32)).to(dtype).cuda()
    for at in range(33):
        _check(flat[at:at + 5 * V].view(5, V), _tokens(rng, (5,), V), 1.0, 3)


def test_a_pointer_between_elements_is_refused():
    z = torch.zeros(64, device="cuda")
    t, out = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, device="cuda")
    for dtype, off in ((sd.SD_F32, 2), (sd.SD_F32, 1), (sd.SD_BF16, 1)):
        status = sd.lib().sd_token_logprobs(z.data_ptr() + off, dtype, 2, 8, 8, t.data_ptr(), 1.0, 0, out.data_ptr(),
                                            None, None, None, None)
        assert status == 1
