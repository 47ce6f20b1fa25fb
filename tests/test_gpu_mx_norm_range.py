"""The norm at the ends of binary32: rows so small or so large that the factor itself, or its size, is no normal number of 32 bits."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2103_14949_amd as hago
import test_gpu_mx as t
from oracle import mx_ref as mx


@pytest.mark.parametrize("cols", [33, 200, 1283, 4100, 33000])
@pytest.mark.parametrize("name,fmt", [("f32", "fp8"), ("f32", "fp4"), ("bf16", "fp8")])
@pytest.mark.parametrize("with_gamma", [False, True])
def test_rows_of_any_size_without_eps(cols, name, fmt, with_gamma):
    """eps = 0: the norm does not depend on a row's size.  Rows of magnitudes from 2^-140 (bf16, which ends at 2^-133: 2^-131) to 2^126;
    subnormal numbers have fewer bits, but exact ones."""
    gen = torch.Generator().manual_seed(cols)
    sizes = [-140, -135, -130, -128, -127, -126, -125, -120, -101, -99, -30, 0, 30, 99, 101, 120, 124, 125]
    sizes = [e for e in sizes if e >= (-140 if name == "f32" else -131)]
    x = torch.randn(len(sizes), cols, generator=gen).clamp(-3.9, 3.9)
    x = torch.from_numpy(np.ldexp(x.double().numpy(), np.array(sizes)[:, None])).to(t.TYPES[name])
    assert int((x != 0).sum(1).min()) > 0
    gamma = (1 + 0.3 * torch.randn(cols, generator=gen)).to(t.TYPES[name]) if with_gamma else None
    got, values = hago.mx_rmsnorm(x.to(t.DEV), None if gamma is None else gamma.to(t.DEV), eps=0.0, fmt=t.FORMATS[fmt], values=True)
    y = mx.rmsnorm(x.double().numpy(), None if gamma is None else gamma.double().numpy(), eps=0.0)[1]
    codes, scales = t.host(got.codes), t.host(got.scales)
    assert [e for row, e in enumerate(sizes) if not mx.accepts(codes[row:row + 1], scales[row:row + 1], y[row:row + 1], t.NORM_DELTA, fmt)] == []
    assert t.same_values(values, mx.decode(codes, scales, fmt, cols), t.TYPES[name])


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_gammas_that_bring_a_row_back(fmt):
    """A row of one large number and small ones, whose norm gamma raises again: products of factor and gamma, each far from 1."""
    cols = 256
    x = torch.full((2, cols), 1.0)
    x[0, 0], x[1, 0] = 2.0 ** 110, 2.0 ** 60
    gamma = torch.full((cols,), 2.0 ** 100) * (1 + torch.rand(cols, generator=torch.Generator().manual_seed(1)))
    gamma[0] = 1.0
    got = hago.mx_rmsnorm(x.to(t.DEV), gamma.to(t.DEV), eps=0.0, fmt=t.FORMATS[fmt])
    y = mx.rmsnorm(x.double().numpy(), gamma.double().numpy(), eps=0.0)[1]
    assert mx.accepts(t.host(got.codes), t.host(got.scales), y, t.NORM_DELTA, fmt)


@pytest.mark.parametrize("cols", [1, 33, 300, 1100, 8200, 16400, 33000])
@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_a_row_that_is_no_number_leaves_the_room_behind_it_empty(cols, fmt):
    """Blocks without a column keep zero codes and the scale byte 0, whatever the row holds (a NaN, or zeros without eps)."""
    x = torch.randn(4, cols, generator=torch.Generator().manual_seed(2))
    x[1, cols // 2], x[3] = float("nan"), 0.0
    gamma = torch.ones(cols)
    for g in (None, gamma):
        got = hago.mx_rmsnorm(x.to(t.DEV), None if g is None else g.to(t.DEV), eps=0.0, fmt=t.FORMATS[fmt])
        want = np.full((2, cols), np.nan)
        codes, scales = mx.encode(want, fmt)
        assert np.array_equal(t.host(got.scales)[[1, 3]], scales) and np.array_equal(t.host(got.codes)[[1, 3]], codes)
