"""Appends under the largest scales."""
import numpy as np
import pytest
import torch

import oracle
from paper_2606_31160_gb300 import sd, workloads
from tests.helpers import ensure_lib, to64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_lib()
    sd.get_device_error()


def _codes(t):
    return t.float().cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("e", [100, 125, 126, 127])
def test_append_under_a_large_scale(e):
    """Any positive scale may stand in a block that holds rows, up to the largest power of
    two: the code is the value over it."""
    c = sd.KV8Cache.empty(1, 1, 64, 64, 64)
    c.k_scale.fill_(2.0 ** e)
    c.v_scale.fill_(2.0 ** e)
    c.len.fill_(3)
    new = np.zeros((1, 2, 1, 64), dtype=np.float32)
    new[0, 0, 0, :5] = np.float32(2.0 ** e) * np.array([1.0, -1.5, 1.9921875, 0.125, 0.0], dtype=np.float32)
    new = workloads.to_bf16(new).cuda()
    sd.kv8_append(c, new, new)
    want = oracle.round_e4m3(to64(new)[0, :, 0] / 2.0 ** e)
    for t in (c.k, c.v):
        assert np.array_equal(_codes(t)[0, 0, 3:5], want)
    assert c.k_scale.item() == 2.0 ** e and sd.get_device_error() == 0
