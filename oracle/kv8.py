"""The 8-bit KV cache (test infrastructure, oracle only).

A value is code * scale: the code an e4m3 number (sign, 4 exponent bits of bias 7, 3
mantissa bits, no infinities, largest 448), the scale one number for each block of
consecutive tokens of a KV head. A block that begins with new rows takes the smallest
power of two, at least 2^-100, that keeps its largest finite magnitude within 448; a
block with older rows keeps its scale times the least power of two (1 or more) that fits
the new ones, and the older codes are rounded anew under it.

Parity: pinned (tests/test_oracle_kv8.py) by the list of all 256 codes, by torch's
float8_e4m3fn conversion, and by the error bound of a 4-bit significand.
"""

import numpy as np

E4M3_MAX = 448.0
MIN_EXP = -100


def e4m3_values():
    """The 256 values of the codes 0 .. 255 (NaN at 0x7f and 0xff)."""
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = np.nan if (e, m) == (15, 7) else (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
        out[c] = -x if c & 128 else x
    return out


_GRID = np.sort(e4m3_values()[:127])  # the non-negative numbers


def round_e4m3(x):
    """The nearest e4m3 number, ties to the even mantissa; infinities saturate, NaN stays."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.abs(x), E4M3_MAX)
    hi = np.minimum(np.searchsorted(_GRID, np.nan_to_num(a)), len(_GRID) - 1)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - _GRID[lo], _GRID[hi] - a
    pick = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)  # the grid's index has its code's parity
    return np.where(np.isnan(x), np.nan, np.copysign(_GRID[pick], x))


def block_scale(rows):
    """Scale of a block that holds these rows and no older ones."""
    a = np.abs(rows[np.isfinite(rows)])
    amax = a.max() if a.size else 0.0
    e = MIN_EXP
    while amax > E4M3_MAX * 2.0 ** e:
        e += 1
    return 2.0 ** e


def kv8_append(codes, scales, lens, new, block):
    """Append new [B, R, H, D] to codes (as values) [B, H, cap, D] with scales
    [B, H, nblk] at lens [B]; returns new (codes, scales). Scenes past the capacity raise."""
    codes, scales = np.array(codes, dtype=np.float64), np.array(scales, dtype=np.float64)
    B, R, H, _ = new.shape
    for b in range(B):
        n0 = int(lens[b])
        if n0 + R > codes.shape[2]:
            raise ValueError("append beyond capacity")
        for h in range(H):
            for blk in range(n0 // block, (n0 + R - 1) // block + 1):
                lo, hi = max(blk * block, n0), min((blk + 1) * block, n0 + R)
                rows = new[b, lo - n0:hi - n0, h]
                if lo == blk * block:
                    s = block_scale(rows)
                else:
                    s = scales[b, h, blk]
                    a = np.abs(rows[np.isfinite(rows)])
                    g = 0
                    while a.size and a.max() > E4M3_MAX * s * 2.0 ** g:
                        g += 1
                    s = s * 2.0 ** g
                    codes[b, h, blk * block:lo] = round_e4m3(codes[b, h, blk * block:lo] * 2.0 ** -g)
                scales[b, h, blk] = s
                codes[b, h, lo:hi] = round_e4m3(rows / s)
    return codes, scales


def dequantise(codes, scales, block):
    """Values [B, H, cap, D] that codes and block scales stand for."""
    n = codes.shape[2]
    return codes * np.repeat(scales, block, axis=2)[:, :, :n, None]
