"""The sign of zero through the norm and the activation: codes of -0 are not those of +0 (include/hago.h)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2103_14949_amd as hago
import test_gpu_mx as t
from oracle import mx_ref as mx


def signs(got, fmt):
    codes = mx.unpack(t.host(got.codes), fmt)
    return codes >= (8 if fmt == "fp4" else 128), codes % (8 if fmt == "fp4" else 128) == 0


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_activation(name, fmt):
    gate = torch.tensor([0.0, -0.0, 0.0, -0.0, 1.0, -1.0, 1.0, -1.0] * 4)
    up = torch.tensor([1.0, 1.0, -1.0, -1.0, 0.0, 0.0, -0.0, -0.0] * 4)
    x = torch.cat([gate, up])[None].to(t.TYPES[name])
    got, values = hago.mx_silu_mul(x.to(t.DEV), t.FORMATS[fmt], values=True)
    want = np.signbit(mx.silu_mul(x.double().numpy()))
    negative, zero = signs(got, fmt)
    assert zero.all() and np.array_equal(negative[:, :32], want) and not negative[:, 32:].any()
    assert np.array_equal(np.signbit(t.wide(values)), want)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("cols", [60, 1000, 40000])
def test_norm(cols, name, fmt):
    gen = torch.Generator().manual_seed(cols)
    x = torch.randn(3, cols, generator=gen)
    x[:, ::3], x[:, 1::6] = 0.0, -0.0
    x = (x * torch.tensor([[1.0], [2.0 ** -110], [2.0 ** 60]])).to(t.TYPES[name])
    gamma = (torch.rand(cols, generator=gen) + 0.5) * torch.where(torch.rand(cols, generator=gen) < 0.5, -1.0, 1.0)
    gamma = gamma.to(t.TYPES[name])
    for g in (None, gamma):
        got, values = hago.mx_rmsnorm(x.to(t.DEV), None if g is None else g.to(t.DEV), eps=0.0, fmt=t.FORMATS[fmt], values=True)
        y = mx.rmsnorm(x.double().numpy(), None if g is None else g.double().numpy(), eps=0.0)[1]
        negative, _ = signs(got, fmt)
        assert np.array_equal(negative[:, :cols], np.signbit(y)) and not negative[:, cols:].any()
        assert np.array_equal(np.signbit(t.wide(values)), np.signbit(y))
