"""The operators around the cache together with the products, as the example serves a layer of attention."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import mx_attention_layer as example  # noqa: E402


@pytest.mark.parametrize("width,heads,kv_heads,dim,page,lengths", [(256, 4, 2, 64, 16, (37, 5)), (320, 6, 1, 32, 5, (90,)), (512, 4, 4, 128, 64, (130, 1, 64))])
def test_the_layer_is_near_the_one_in_32_bits(width, heads, kv_heads, dim, page, lengths):
    """Rounding to 4-bit weights and values (2^-2 at most, an eighth on the average) and to 8-bit activations leaves two products and an average within 0.4 of the result, where a
    wrong row, head, page or position leaves 1 and more.  In any steps the layer is the same function of the same codes, but for the order of
    sums and the codes behind them, which may fall to the other side of a rounding."""
    weights = example.make(width, heads, kv_heads, dim, seed=dim)
    gen = torch.Generator(device="cuda").manual_seed(page)
    xs, residuals = ([torch.randn(n, width, generator=gen, device="cuda").bfloat16() for n in lengths] for _ in range(2))
    whole = example.serve(weights, heads, kv_heads, xs, residuals, [[n] for n in lengths], page)
    steps = example.serve(weights, heads, kv_heads, xs, residuals, [[n // 3, n // 3, n - n // 4] + list(range(n - n // 4 + 1, n + 1)) + [n] * (max(lengths) // 4 - n // 4)
                                                                   for n in lengths], page)
    for out, again, x, r in zip(whole, steps, xs, residuals):
        want, _ = example.plain(weights, x, r, heads, kv_heads)
        assert out.dtype == torch.bfloat16 and (out.float() - want).norm() < 0.4 * want.norm()
        assert (again.float() - out.float()).norm() < 0.05 * out.float().norm()
