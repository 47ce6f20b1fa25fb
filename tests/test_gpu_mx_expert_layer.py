"""The microscaled operators together, as the example serves a layer of experts."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import mx_expert_layer as example  # noqa: E402


@pytest.mark.parametrize("tokens,experts,width,hidden,top", [(1, 4, 256, 192, 2), (37, 8, 320, 96, 3), (300, 5, 512, 257, 1), (64, 16, 1024, 704, 4)])
def test_the_layer_is_near_the_one_in_32_bits(tokens, experts, width, hidden, top):
    """Rounding to 4-bit codes leaves 2^-2 at most and an eighth or so on the average of a weight, which random rows average out no
    further than their own norms: two products of 4-bit weights and 8-bit activations (2^-4 at most) stay within 0.3 of the result,
    where a wrong row, expert or weight leaves 1 and more.  Tokens that the two forms route differently (near ties) are left out."""
    weights = example.make(experts, width, hidden, seed=tokens)
    layer = example.ExpertLayer(*weights, top)
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    x, residual = (torch.randn(tokens, width, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    out, new = layer(x, residual)
    want, h = example.plain(weights, x, residual, top)
    assert out.dtype == torch.bfloat16 and torch.equal(new, h.to(torch.bfloat16))
    off = (out.float() - want).norm(dim=1) / want.norm(dim=1)
    assert float(off.median()) < 0.3 and float((off < 0.5).float().mean()) > 0.8
    again = layer(x, residual)
    assert torch.equal(again[0], out) and torch.equal(again[1], new)
