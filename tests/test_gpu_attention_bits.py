"""What bfloat16 calls of the attention lose: beside the rounding of the result, nothing that its bits could show."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2103_14949_amd as hago
from cache_util import DEV, check_attention, layout, on_gpu, random_cache
from oracle import cache_ref as ref


def half_step(x):
    """Half a step of bfloat16's at |x|: eight bits from the leading one on."""
    return np.exp2(np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -126))) - 8)


def off(new, lengths, heads, kv_heads, dim, seed, probability, k_fmt="fp8", v_fmt="fp8", page=16, edit=None, **call):
    """A result is the sum over the keys, rounded once: half a step of the value before, which is off by the share of sum p |v| that cache_util.attention_bound counts:
    2^-24 of the scores' magnitudes and 2^-22 of the exponent twice, 2^-24 a key, and `probability`, by which a probability in the second product is rounded.  Probabilities
    below 2^-27 of the largest lose up to 2^-38 of that, where they are rounded to float16's 2^-11."""
    rng = np.random.default_rng(seed)
    table, lengths, offsets, pages = layout(new, lengths, page, seed=seed)
    cache, keys, values = random_cache(rng, pages, kv_heads, page, dim, k_fmt, v_fmt)
    if edit:
        edit(rng, cache, values)
    q = torch.from_numpy(rng.standard_normal((int(offsets[-1]), heads, dim))).to(torch.bfloat16)
    got = hago.mx_attention(q.to(DEV), cache, *on_gpu(table, lengths, offsets), **call).double().cpu().numpy()
    out, _, weight, spread = ref.attention(q.double().numpy(), keys, values, ref.Sequences(table, lengths, offsets, pages, page), dim ** -0.5, **call)
    score = (dim + 4) * 2.0 ** -24 * spread + 2.0 ** -22 * (spread + 1)
    before = weight * (probability + 2 * (max(lengths) + 64) * 2.0 ** -24 + 2 * score)[..., None]
    if probability == 2.0 ** -11:
        before = before + max(lengths) * 2.0 ** -38 * np.abs(values).max((0, 1, 2))
    return np.abs(got - out) / (before + half_step(np.abs(out) + before))


@pytest.mark.parametrize("dim", [40, 64, 128, 256])
@pytest.mark.parametrize("new,lengths", [([1, 1], [3, 40]), ([4, 2, 1], [4, 600, 33]), ([1], [5000])])
def test_few_rows(new, lengths, dim):
    """Probabilities of two bfloat16 numbers: 2^-16."""
    assert off(new, lengths, 8, 4, dim, dim, 2.0 ** -16).max() <= 1


@pytest.mark.parametrize("k_fmt,v_fmt", [("fp8", "fp8"), ("fp4", "fp4"), ("fp4", "fp8")])
@pytest.mark.parametrize("dim", [3, 40, 64, 96, 128])
@pytest.mark.parametrize("new,lengths", [([70, 9], [70, 40]), ([33, 40], [700, 33]), ([40], [5000])])
def test_many_rows(new, lengths, dim, k_fmt, v_fmt):
    """Probabilities of one float16 number: 2^-11."""
    assert off(new, lengths, 8, 4, dim, dim, 2.0 ** -11, k_fmt, v_fmt).max() <= 1


def scaled(cache, values, where, by):
    """Blocks `where` [pages, kv_heads, page, blocks] of the values 2^by times theirs."""
    cache.v_scales += torch.from_numpy(np.where(where, by, 0).astype(np.int8)).to(DEV).view(torch.uint8)   # (modulo 256)
    whole = np.repeat(where, 32, -1)[..., :values.shape[-1]]
    values[whole] *= 2.0 ** by


@pytest.mark.parametrize("page", [16, 20])
@pytest.mark.parametrize("v_fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("dim", [40, 64, 128])
@pytest.mark.parametrize("by", [-100, -40, -16, 14, 40, 100])
def test_values_beyond_float16(by, dim, v_fmt, page):
    """Blocks that float16 does not hold, in few tokens and in most, among others that it does; and blocks of zeros."""
    for share in (0.003, 0.5, 1.0):
        def edit(rng, cache, values):
            where = rng.random(cache.v_scales.shape) < share
            scaled(cache, values, where, by)
            zero = rng.random(cache.v_scales.shape) < 0.2
            whole = torch.from_numpy(np.repeat(zero, cache.v_codes.shape[-1] // zero.shape[-1], -1)).to(DEV)
            cache.v_codes[whole] = 0
            cache.v_scales[torch.from_numpy(zero).to(DEV)] = 0
            values[np.repeat(zero, 32, -1)[..., :dim]] = 0
        assert off([70, 50], [300, 90], 2, 1, dim, dim + 3, 2.0 ** -11, "fp8", v_fmt, page, edit).max() <= 1
    assert off([70], [4000], 2, 2, dim, dim + 5, 2.0 ** -11, "fp8", v_fmt, page, lambda rng, cache, values: scaled(cache, values, rng.random(cache.v_scales.shape) < 0.001, by),
               window=2000).max() <= 1


@pytest.mark.parametrize("fmt,codes", [("fp8", range(127)), ("fp4", range(8))])
@pytest.mark.parametrize("up", [0, 1])
def test_every_code_at_the_ends_of_float16(up, fmt, codes):
    """A row that sees one token, whose block has each code in turn, at the scales next to where the kernel turns from one form of values to the other: the value itself."""
    dim, kept = 128, list(codes)
    for byte in {"fp8": (107 - up, 129 + up), "fp4": (99 - up, 135 + up)}[fmt]:
        tokens = -(-len(kept) // 128) * 64
        cache = hago.MXCache.empty(tokens // 16, 1, 16, dim, hago.MX_FP8, hago.MX_FP8 if fmt == "fp8" else hago.MX_FP4)
        cache.k_codes.zero_(), cache.k_scales.fill_(127), cache.v_scales.fill_(byte)
        raw = torch.arange(cache.v_codes.numel()) * 7 % (len(kept) if fmt == "fp8" else 256)
        cache.v_codes.copy_(raw.to(torch.uint8).view(cache.v_codes.shape))
        where = on_gpu(np.arange(tokens // 16, dtype=np.int32)[None], np.array([tokens], np.int32), np.array([0, tokens], np.int32))
        q = torch.zeros(tokens, 1, dim, dtype=torch.bfloat16, device=DEV)
        got = hago.mx_attention(q, cache, *where, window=1)
        want = hago.mx_cache_read(cache, *where, tokens, out_dtype=hago.BF16)[1]
        assert torch.equal(got, want)


def test_none_and_beyond_float16_together():
    """A block of NaN beside blocks that float16 does not hold, and bytes that nobody wrote behind the last token: as in test_what_is_hidden_is_not_seen."""
    rng = np.random.default_rng(4)
    table, lengths, offsets, pages = layout([150], [200], 16)
    cache, keys, values = random_cache(rng, pages, 1, 16, 128, "fp8", "fp8")
    scaled(cache, values, rng.random(cache.v_scales.shape) < 0.1, -30)
    seqs = ref.Sequences(table, lengths, offsets, pages, 16)
    for page, at in {(p, a) for p in range(pages) for a in range(16)} - {seqs.place(0, j) for j in range(200)}:
        for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales):
            t[page, 0, at] = 0xFF
    q = torch.from_numpy(rng.standard_normal((150, 2, 128))).to(torch.bfloat16)
    where = on_gpu(table, lengths, offsets)
    want = hago.mx_attention(q.to(DEV), cache, *where)
    check_attention(want, "bf16", q.double().numpy(), keys, values, seqs, 128 ** -0.5)
    page, at = seqs.place(0, 120)   # row 70 is the first that sees it
    cache.v_scales[page, 0, at, 1] = 255
    got = hago.mx_attention(q.to(DEV), cache, *where)
    assert got[70:, :, 32:64].isnan().all() and torch.equal(got[:70], want[:70])
    other = [c for c in range(128) if not 32 <= c < 64]
    assert torch.equal(got[:, :, other], want[:, :, other])


@pytest.mark.parametrize("dim", [129, 200, 256])
@pytest.mark.parametrize("new,lengths", [([70, 9], [70, 40]), ([33, 40], [700, 33]), ([40], [5000])])
def test_many_rows_of_more_than_128_columns(new, lengths, dim):
    """Two bfloat16 numbers in the kernel for many rows: 2^-16."""
    assert off(new, lengths, 8, 4, dim, dim, 2.0 ** -16).max() <= 1


@pytest.mark.parametrize("v_fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("sign", [0, 1])
@pytest.mark.parametrize("byte", [0, 1, 128, 200, 245, 249, 250, 251, 254])
def test_zeros_of_any_scale(byte, sign, v_fmt):
    """A block of zeros, of either sign, stands for zeros whatever its scale is; a quarter of a block, too."""
    rng = np.random.default_rng(byte)
    table, lengths, offsets, pages = layout([70], [200], 16)
    cache, keys, values = random_cache(rng, pages, 1, 16, 128, "fp8", v_fmt)
    code = (0x88 if v_fmt == "fp4" else 0x80) if sign else 0
    where = rng.random(cache.v_scales.shape) < 0.3
    cache.v_scales[torch.from_numpy(where).to(DEV)] = byte
    cache.v_codes[torch.from_numpy(np.repeat(where, cache.v_codes.shape[-1] // where.shape[-1], -1)).to(DEV)] = code
    values[np.repeat(where, 32, -1)] = 0
    q = torch.from_numpy(rng.standard_normal((70, 2, 128))).to(torch.bfloat16)
    out = hago.mx_attention(q.to(DEV), cache, *on_gpu(table, lengths, offsets))
    check_attention(out, "bf16", q.double().numpy(), keys, values, ref.Sequences(table, lengths, offsets, pages, 16), 128 ** -0.5)
