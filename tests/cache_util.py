"""Paged caches and batches of sequences for the tests of the operators around them."""
import numpy as np
import torch

import paper_2103_14949_amd as hago
from oracle import cache_ref as ref

DEV = "cuda:0"
FORMATS = {"fp4": hago.MX_FP4, "fp8": hago.MX_FP8}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
OUT = {"f32": hago.F32, "bf16": hago.BF16, "f16": hago.F16}


def layout(new, lengths, page, seed=0, spare=2, extra=1, rows_before=0):
    """Pages in random order: (table, lengths, offsets, pages) in numpy."""
    rng = np.random.default_rng(seed)
    need = [max(0, -(-n // page)) for n in lengths]
    pages = sum(need) + spare
    order = rng.permutation(pages).astype(np.int32)
    table = rng.integers(-3, pages + 3, (len(new), max(need + [0]) + extra)).astype(np.int32)   # entries behind a sequence's end may be anything
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    offsets = np.concatenate([[0], np.cumsum(new)]).astype(np.int32) + rows_before
    return table, np.array(lengths, np.int32), offsets.astype(np.int32), pages


def random_cache(rng, pages, kv_heads, page, dim, k_fmt, v_fmt):
    """(MXCache on the GPU, its keys and values in 64 bits [pages, kv_heads, page, dim])."""
    parts, real = [], []
    for fmt, gain in ((k_fmt, 1.5), (v_fmt, 1.0)):
        x = rng.standard_normal((pages * kv_heads * page, dim)) * gain * np.exp2(rng.integers(-2, 3, (1, dim)))
        codes, scales = ref.encode_row(x, fmt)
        real.append(ref.decode_row(codes, scales, fmt, dim).reshape(pages, kv_heads, page, dim))
        parts += [torch.from_numpy(c.reshape(pages, kv_heads, page, -1).copy()).to(DEV) for c in (codes, scales)]
    return hago.MXCache(*parts, FORMATS[k_fmt], FORMATS[v_fmt], dim), *real


def on_gpu(*arrays):
    return tuple(torch.from_numpy(np.ascontiguousarray(a)).to(DEV) for a in arrays)


def attention_bound(name, out, weight, spread, keys, dim):
    """How far a row may be off.  Scores are sums of `dim` exact products in binary32 (2^-24 of the sum of their magnitudes each), scaled and
    exponentiated (2^-22 of their size and 1 in all): `score` is the relative error of a probability.  Probabilities go into the
    product in one, two or three bfloat16 numbers (2^-8, 2^-16, 2^-24 of them).  The sums over the keys and the running factors add 2^-24 a key
    and as much a block, above and below the line; the result is rounded once."""
    u = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}[name]
    pieces = {"bf16": 2.0 ** -8, "f16": 2.0 ** -16, "f32": 2.0 ** -24}[name]
    score = (dim + 4) * 2.0 ** -24 * spread + 2.0 ** -22 * (spread + 1)
    share = pieces + 2 * (keys + 64) * 2.0 ** -24 + 2 * score
    return weight * share[..., None] * (1 + u) + u * np.abs(out) + (2.0 ** -25 if name == "f16" else 0)   # (float16's smallest step is 2^-24)


def check_attention(got, name, q, keys, values, seqs, scale, causal=True, window=0, lse=None):
    out, want_lse, weight, spread = ref.attention(q, keys, values, seqs, scale, causal, window)
    inside = ~np.isnan(out).all(-1)
    longest = max([0] + [int(n) for n in seqs.lengths])
    bound = attention_bound(name, out, weight, spread, longest, q.shape[2])
    got = got.double().cpu().numpy()
    off = np.abs(got - out)[inside]
    assert not np.isnan(off).any()
    assert (off <= bound[inside]).all(), float((off / bound[inside]).max())
    if lse is not None:
        lse = lse.double().cpu().numpy()[inside]
        want = want_lse[inside]
        empty = np.isneginf(want)
        assert (np.isneginf(lse) == empty).all()
        limit = (q.shape[2] + 8) * 2.0 ** -24 * spread[inside] + 2.0 ** -21 * (np.abs(want) + 1) + 2 * (longest + 64) * 2.0 ** -24
        assert (np.abs(lse[~empty] - want[~empty]) <= limit[~empty]).all()
    return out, inside
