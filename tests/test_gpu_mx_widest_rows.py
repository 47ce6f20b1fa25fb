"""Operators by rows at the widest row that they take, 2^31 - 129 columns."""
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2103_14949_amd as hago

DEV = "cuda:0"
COLS = 2 ** 31 - 129


def holds(got, cols, code, scale):
    """Every column has this code (a byte of codes), every block of columns this scale, nothing behind them."""
    codes, scales = got.codes[0], got.scales[0]
    per_byte = 2 if got.fmt == hago.MX_FP4 else 1
    whole, blocks = cols // per_byte, -(-cols // 32)
    assert bool((codes[:whole] == code).all()) and bool((scales[:blocks] == scale).all()) and bool((scales[blocks:] == 0).all())
    tail = codes[whole:].tolist()
    assert tail == ([code & 15] + [0] * (len(tail) - 1) if cols % per_byte else [0] * len(tail))


@pytest.mark.timeout(120)
def test_the_widest_row():
    x = torch.ones(1, COLS, dtype=torch.bfloat16, device=DEV)
    holds(hago.mx_quantize(x, hago.MX_FP4), COLS, 0x66, 125)     # 1 = 4 * 2^-2
    holds(hago.mx_rmsnorm(x, eps=0.0), COLS, 0x78, 119)          # 1 = 256 * 2^-8
    half = (COLS - 1) // 2
    x[0, :half] = 100.0                                         # silu(100) = 100, times 1: 400 * 2^-2, a tie of 384 (even) and 416
    holds(hago.mx_silu_mul(x[:, :2 * half], hago.MX_FP8), half, 0x7C, 125)
