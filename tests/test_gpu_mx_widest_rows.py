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


@pytest.mark.timeout(120)
@pytest.mark.parametrize("name", ["quantize", "rmsnorm", "silu_mul"])
def test_the_longest_column(name):
    """So many rows that one launch does not hold their threads: the rows on either side of where the next begins, and the last ones."""
    rows, cols = (1 << 28) + 37, 3
    torch.cuda.empty_cache()
    call = {"quantize": lambda x, **k: hago.mx_quantize(x, hago.MX_FP4, **k), "rmsnorm": lambda x, **k: hago.mx_rmsnorm(x, fmt=hago.MX_FP4, **k),
            "silu_mul": lambda x, **k: hago.mx_silu_mul(x, hago.MX_FP4, **k)}[name]
    wide = cols * (2 if name == "silu_mul" else 1)
    x = torch.ones(rows, wide, dtype=torch.bfloat16, device=DEV)
    x[-80:] = torch.randn(80, wide, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(DEV)
    out = hago.MX.empty(rows, cols, hago.MX_FP4, DEV)
    out.codes.fill_(0xA5), out.scales.fill_(0xA5)
    got, one = call(x, out=out), call(x[:1])
    tail = call(x[-80:].contiguous())
    assert torch.equal(got.codes[-80:], tail.codes) and torch.equal(got.scales[-80:], tail.scales)
    for part, scales in zip(got.codes[:-80].split(1 << 24), got.scales[:-80].split(1 << 24)):
        assert bool((part == one.codes).all()) and bool((scales == one.scales).all())
    torch.cuda.empty_cache()
