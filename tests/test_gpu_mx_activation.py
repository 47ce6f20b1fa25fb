"""The gated activation where normal numbers do not reach.

Each against the oracle in 64 bits, with the bound of test_gpu_mx (SILU_DELTA); gates and products are normal numbers of binary32."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2103_14949_amd as hago
import test_gpu_mx as t
from oracle import mx_ref as mx


def check(x, fmt, spoiled=()):
    """x [rows, 2 cols] through the operator.  spoiled: (row, block) that have to stand for NaN; no other one may."""
    cols = x.shape[1] // 2
    got, values = hago.mx_silu_mul(x.to(t.DEV), t.FORMATS[fmt], values=True)
    codes, scales = t.host(got.codes), t.host(got.scales)
    with np.errstate(over="ignore", invalid="ignore"):
        y = mx.silu_mul(x.double().numpy())
    wide = np.zeros((len(y), mx.padded(cols)))
    wide[:, :cols] = y
    blocks = wide.reshape(len(y), -1, 32)
    bad = np.zeros(blocks.shape[:2], bool)
    for row, block in spoiled:
        bad[row, block] = True
    assert np.array_equal(scales == 255, bad)
    per_block = codes.reshape(*bad.shape, -1)
    assert (per_block[bad] == 0).all()
    blocks[bad] = 0
    scales = np.where(bad, 0, scales).astype(np.uint8)
    assert mx.accepts(codes, scales, blocks.reshape(wide.shape)[:, :cols], t.SILU_DELTA, fmt)
    decoded = mx.decode(codes, np.where(bad, 255, scales), fmt, cols)
    assert t.same_values(values, decoded, x.dtype)


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_a_gate_or_an_up_that_is_no_number_spoils_its_block_alone(name, fmt):
    nan, inf = float("nan"), float("inf")
    cols = 300
    x = torch.randn(8, 2 * cols, generator=torch.Generator().manual_seed(3)).to(t.TYPES[name])
    spoiled = []
    for row, (at, gate, up) in enumerate([(0, nan, None), (37, inf, None), (299, nan, 0.0), (130, inf, 0.0), (64, None, nan), (95, None, inf), (200, None, -inf), (255, 0.0, inf)]):
        if gate is not None:
            x[row, at] = gate
        if up is not None:
            x[row, cols + at] = up
        spoiled.append((row, at // 32))
    check(x, fmt, spoiled)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_gates_of_every_exponent(name, fmt):
    """A row of gates for every exponent whose half is a normal number, of either sign, times ups that bring the products between 2^-10 and 2^10."""
    gen = torch.Generator().manual_seed(5)
    exponents = range(-125, 6)
    rows = []
    for e in exponents:
        gate = torch.ldexp(1 + torch.rand(96, generator=gen), torch.tensor(e)) * torch.where(torch.rand(96, generator=gen) < 0.5, -1.0, 1.0)
        up = torch.ldexp(1 + torch.rand(96, generator=gen), torch.tensor(min(-e, 120)))
        rows.append(torch.cat([gate, up]))
    check(torch.stack(rows).to(t.TYPES[name]), fmt)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_gates_far_below_zero(name, fmt):
    """Gates from -60 on down, times the largest ups, as long as the products are normal numbers; each with its own small neighbours and with
    neighbours that leave it a zero; and the last finite one."""
    gen = torch.Generator().manual_seed(6)
    rows = []
    for g in [*range(-60, -172, -2), -79.75, -80.5, -88.5, -88.75, -103.5]:
        gate = torch.full((64,), float(g))
        up = torch.ldexp(1 + torch.rand(64, generator=gen), torch.tensor(126)) * torch.where(torch.rand(64, generator=gen) < 0.5, -1.0, 1.0)
        gate[32] = 1.0
        rows.append(torch.cat([gate, up]))
    x = torch.stack(rows).to(t.TYPES[name])
    x[-1, 40], x[-1, 41], x[-1, 42] = -1e4, torch.finfo(t.TYPES[name]).min, -1000.0
    check(x, fmt)


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_a_gate_of_minus_infinity_is_no_number(fmt):
    """By the formula: minus infinity by infinity."""
    x = torch.randn(3, 200, generator=torch.Generator().manual_seed(7))
    x[1, 5] = -float("inf")
    check(x, fmt, [(1, 0)])
