"""The oracle of the microscaled operators, in numpy and 64 bits (TEST INFRASTRUCTURE ONLY; shares no code with the library).

Formats: "fp4" (E2M1) and "fp8" (E4M3), blocks of 32 columns, scale bytes E8M0, rows in whole blocks of 128 columns.
"""
from __future__ import annotations

import numpy as np

EMAX = {"fp4": 2, "fp8": 8}


def code_values(fmt):
    """The value of every code by its bits: sign, exponent, mantissa (NaN where the code is none)."""
    bits, ebits, mbits, bias = (4, 2, 1, 1) if fmt == "fp4" else (8, 4, 3, 7)
    v = np.empty(1 << bits)
    for c in range(1 << bits):
        m = c & ((1 << mbits) - 1)
        e = c >> mbits & ((1 << ebits) - 1)
        size = (1 + m / (1 << mbits)) * 2.0 ** (e - bias) if e else m / (1 << mbits) * 2.0 ** (1 - bias)
        if fmt == "fp8" and c & 127 == 127:
            size = np.nan
        v[c] = -size if c >> (bits - 1) else size
    return v


def padded(cols):
    return -(-cols // 128) * 128


def pack(codes, fmt):
    """Codes, one a byte -> as they lie in memory."""
    codes = codes.astype(np.uint8)
    return codes if fmt == "fp8" else codes[..., 0::2] | codes[..., 1::2] << 4


def unpack(codes, fmt):
    return codes if fmt == "fp8" else np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1])


def decode(codes, scales, fmt, cols):
    """Codes as they lie in memory and scale bytes -> values [..., cols] in 64 bits."""
    scale = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (code_values(fmt)[unpack(codes, fmt)] * np.repeat(scale, 32, -1))[..., :cols]


def nearest_codes(scaled, fmt):
    """Magnitude codes nearest to |scaled|, ties to the even code, saturating; by comparison with every midpoint."""
    grid = code_values(fmt)[:8 if fmt == "fp4" else 127]
    mid = (grid[1:] + grid[:-1]) / 2
    a = np.abs(scaled)
    low = np.searchsorted(mid, a, side="left")      # ties: the lower code
    high = np.searchsorted(mid, a, side="right")    # ties: the upper code
    return np.where(low % 2 == 0, low, high)


def block_scales(x, fmt):
    """Exponents (of two) of the blocks' scales; x in whole blocks, finite."""
    m = np.abs(x).reshape(*x.shape[:-1], x.shape[-1] // 32, 32).max(-1)
    e = np.frexp(np.where(m > 0, m, 1.0))[1] - 1 - EMAX[fmt]
    return np.maximum(np.where(m > 0, e, -127), -127)


def encode(x, fmt, exponents=None):
    """x [rows, cols] -> (codes as they lie in memory, scale bytes), whole blocks of 128 columns.  exponents: the blocks' scales, where
    they are not to come from x."""
    rows, cols = x.shape
    wide = np.zeros((rows, padded(cols)))
    wide[:, :cols] = x
    blocks = wide.reshape(rows, wide.shape[1] // 32, 32)
    bad = ~np.isfinite(blocks).all(-1)
    clean = np.where(bad[..., None], 0.0, blocks)
    e = block_scales(clean.reshape(wide.shape), fmt) if exponents is None else exponents
    codes = nearest_codes(np.ldexp(clean, -e[..., None]), fmt)
    codes = codes + np.signbit(clean) * (8 if fmt == "fp4" else 128)
    codes = np.where(bad[..., None], 0, codes).astype(np.uint8)
    scales = np.where(bad, 255, e + 127).astype(np.uint8)
    return pack(codes.reshape(wide.shape), fmt), scales


def rmsnorm(x, gamma=None, residual=None, eps=1e-5):
    """(h, y) in 64 bits."""
    h = x.astype(np.float64)
    if residual is not None:
        h = h + residual.astype(np.float64)
    y = h / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    return h, y if gamma is None else y * gamma.astype(np.float64)


def silu_mul(x):
    g, u = np.split(x.astype(np.float64), 2, -1)
    return g / (1 + np.exp(-g)) * u


def accepts(codes, scales, y, rel, fmt):
    """Whether every block encodes numbers within rel (relative) of y: its scale is one that they can have, and every code lies between
    those of the two ends."""
    rows, cols = y.shape
    wide = np.zeros((rows, padded(cols)))
    wide[:, :cols] = y
    low, high = block_scales(wide * (1 - rel), fmt), block_scales(wide * (1 + rel), fmt)
    e = scales.astype(np.int64) - 127
    if not ((e == low) | (e == high)).all():
        return False
    blocks = wide.reshape(rows, -1, 32)
    got = unpack(codes, fmt).reshape(blocks.shape).astype(np.int64)
    sign = 8 if fmt == "fp4" else 128
    size, negative = got % sign, got >= sign
    lo = nearest_codes(np.ldexp(blocks * (1 - rel), -e[..., None]), fmt)
    hi = nearest_codes(np.ldexp(blocks * (1 + rel), -e[..., None]), fmt)
    return bool(((size >= lo) & (size <= hi) & ((negative == (blocks < 0)) | (size == 0))).all())
