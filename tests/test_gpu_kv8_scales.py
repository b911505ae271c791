"""Appends under the largest scales, and what rejected rows leave of the older codes."""
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


@pytest.mark.parametrize("D,block", [(128, 64), (64, 32)])
def test_what_rejected_rows_leave(D, block):
    """Draft rows that are appended and rolled back, each larger than the one before: the
    block keeps the scale that fitted them, and its older values stay within what that
    scale's codes can hold: 2^-4 of a value (an e4m3 code's rounding), or, of the small ones,
    half a step of 2^-9 of every scale on the way (together less than one step of the last).
    Rows that need no larger scale leave no mark."""
    rng = np.random.default_rng(block)
    H, n = 2, 20
    c = sd.KV8Cache.empty(1, H, block, D, block)
    rows = workloads.to_bf16((rng.standard_normal((1, n, H, D)) * 2.0 ** rng.integers(-8, 1, (1, n, H, D))).astype(np.float32)).cuda()
    sd.kv8_append(c, rows, rows)
    first, scale = c.k.view(torch.uint8).clone(), c.k_scale.clone()
    none = torch.zeros(1, dtype=torch.int32, device="cuda")

    def reject(mag):
        new = rng.standard_normal((1, 3, H, D))
        new = workloads.to_bf16((new / np.abs(new).max() * mag).astype(np.float32)).cuda()
        sd.kv8_append(c, new, new)
        sd.kv_rollback(c.len, none, 3)
    for _ in range(8):
        reject(0.5)
    assert torch.equal(c.k.view(torch.uint8)[:, :, :n], first[:, :, :n]) and torch.equal(c.k_scale, scale)
    for e in range(1, 9):
        reject(4.0 * 2.0 ** e)
    assert c.len.item() == n and (c.k_scale > 50 * scale).all()
    x = to64(rows)[0].transpose(1, 0, 2)
    last = c.k_scale.cpu().numpy().astype(np.float64)[0]
    for t in (c.k, c.v):
        got = oracle.dequantise(_codes(t), c.k_scale.cpu().numpy().astype(np.float64), block)[0, :, :n]
        assert np.all(np.abs(got - x) <= 2.0 ** -4 * np.abs(x) + 2.0 ** -9 * last[:, :, None])
    assert sd.get_device_error() == 0
