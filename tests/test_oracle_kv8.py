"""Pins of the 8-bit cache oracle (oracle/kv8.py)."""
import numpy as np
import torch

import oracle
from oracle.kv8 import block_scale


def test_codes_are_torch_float8():
    mine = oracle.e4m3_values()
    theirs = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(mine, theirs.astype(np.float64), equal_nan=True)


def test_rounding_is_torch_float8():
    rng = np.random.default_rng(0)
    grid = np.unique(np.abs(oracle.e4m3_values()[:127]))
    ties = (grid[1:] + grid[:-1]) / 2
    x = np.concatenate([rng.standard_normal(20000) * 10.0 ** rng.uniform(-4, 2.6, 20000), ties, -ties, grid, [0.0]])
    x = np.clip(x, -448, 448).astype(np.float32)
    assert np.array_equal(oracle.round_e4m3(x), torch.from_numpy(x).to(torch.float8_e4m3fn).float().numpy())
    assert oracle.round_e4m3(np.inf) == 448 and oracle.round_e4m3(-np.inf) == -448 and np.isnan(oracle.round_e4m3(np.nan))


def test_scale_is_the_least_power_of_two():
    for amax in (1e-40, 0.0, 1.0, 1.75, 1.7500001, 448.0, 448.5, 3e38):
        s = block_scale(np.array([amax, -amax / 2, np.inf, np.nan]))
        assert amax <= 448 * s and (s == 2.0 ** -100 or amax > 448 * s / 2)


def test_append_error_and_growth():
    rng = np.random.default_rng(1)
    B, H, cap, D, block = 2, 2, 100, 8, 32
    codes, scales = np.zeros((B, H, cap, D)), np.ones((B, H, 4))
    lens, x = np.array([0, 0]), np.zeros((B, H, cap, D))
    for R, mag in ((5, 1.0), (30, 0.01), (1, 300.0), (40, 1e-3)):
        new = rng.standard_normal((B, R, H, D)) * mag
        codes, scales = oracle.kv8_append(codes, scales, lens, new, block)
        for b in range(B):
            x[b, :, lens[b]:lens[b] + R] = new[b].transpose(1, 0, 2)
        lens = lens + R
    got = oracle.dequantise(codes, scales, block)
    # half a step of a 4-bit significand, or of the subnormals (twice: older codes round again)
    s = np.repeat(scales, block, axis=2)[:, :, :cap, None]
    assert np.all(np.abs(got - x)[:, :, :76] <= (2.0 ** -4 * np.abs(x) + 2.0 ** -9 * s)[:, :, :76])
    assert np.all(codes[:, :, 76:] == 0)
