"""What bfloat16 calls of the attention lose: beside the rounding of the result, nothing that its bits could show."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2103_14949_amd as hago
from cache_util import DEV, layout, on_gpu, random_cache
from oracle import cache_ref as ref


def half_step(x):
    """Half a step of bfloat16's at |x|: eight bits from the leading one on."""
    return np.exp2(np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -126))) - 8)


def off(new, lengths, heads, kv_heads, dim, seed, probability):
    """A result is the sum over the keys, rounded once: half a step of the value before, which is off by the share of sum p |v| that cache_util.attention_bound counts:
    2^-24 of the scores' magnitudes and 2^-22 of the exponent twice, 2^-24 a key, and `probability`, by which a probability in the second product is rounded."""
    rng = np.random.default_rng(seed)
    table, lengths, offsets, pages = layout(new, lengths, 16, seed=seed)
    cache, keys, values = random_cache(rng, pages, kv_heads, 16, dim, "fp8", "fp8")
    q = torch.from_numpy(rng.standard_normal((int(offsets[-1]), heads, dim))).to(torch.bfloat16)
    got = hago.mx_attention(q.to(DEV), cache, *on_gpu(table, lengths, offsets)).double().cpu().numpy()
    out, _, weight, spread = ref.attention(q.double().numpy(), keys, values, ref.Sequences(table, lengths, offsets, pages, 16), dim ** -0.5)
    score = (dim + 4) * 2.0 ** -24 * spread + 2.0 ** -22 * (spread + 1)
    before = weight * (probability + 2 * (max(lengths) + 64) * 2.0 ** -24 + 2 * score)[..., None]
    return np.abs(got - out) / (before + half_step(np.abs(out) + before))


@pytest.mark.parametrize("dim", [40, 64, 128, 256])
@pytest.mark.parametrize("new,lengths", [([1, 1], [3, 40]), ([4, 2, 1], [4, 600, 33]), ([1], [5000])])
def test_few_rows(new, lengths, dim):
    """Probabilities of two bfloat16 numbers: 2^-16."""
    assert off(new, lengths, 8, 4, dim, dim, 2.0 ** -16).max() <= 1


@pytest.mark.parametrize("dim", [129, 200, 256])
@pytest.mark.parametrize("new,lengths", [([70, 9], [70, 40]), ([33, 40], [700, 33]), ([40], [5000])])
def test_many_rows_of_more_than_128_columns(new, lengths, dim):
    """The same in the kernel for many rows."""
    assert off(new, lengths, 8, 4, dim, dim, 2.0 ** -16).max() <= 1
