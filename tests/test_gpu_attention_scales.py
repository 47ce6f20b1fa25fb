"""Scores far from zero: the largest of a row's is the one that counts, whatever the scale, in the kernel for few rows and in the one for many."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2103_14949_amd as hago
from cache_util import DEV, FORMATS, TYPES, layout, on_gpu
from oracle import cache_ref as ref


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("new,length", [(3, 200), (70, 200), (100, 100), (70, 6000)])
@pytest.mark.parametrize("scale", [3e3, 1e5, 1e8, -1e8, 1e9, 1e10, -1e10, 2.0 ** 100, -2.0 ** 100])
def test_the_largest_score_wins(scale, new, length, name):
    """Queries and keys are small whole numbers, so scores are whole numbers that binary32 holds, and every other one is at least |scale| below the largest:
    e^-3000 and less of it.  The row is the average of the values of the keys that have it, each with the same probability, which is what is compared: the sums of n such
    values are off by 2^-24 a term, the probabilities by 2^-22 of their exponent (no more than 6 beyond zero), in two or one bfloat16 numbers by 2^-8 alike for all."""
    rng = np.random.default_rng(length)
    dim, page = 64, 16
    table, lengths, offsets, pages = layout([new], [length], page)
    parts, real = [], []
    for x in (rng.integers(-3, 4, (pages * 2 * page, dim)).astype(np.float64), rng.standard_normal((pages * 2 * page, dim))):
        codes, scales = ref.encode_row(x, "fp8")
        real.append(ref.decode_row(codes, scales, "fp8", dim).reshape(pages, 2, page, dim))
        parts += [torch.from_numpy(c.reshape(pages, 2, page, -1).copy()).to(DEV) for c in (codes, scales)]
    cache = hago.MXCache(*parts, FORMATS["fp8"], FORMATS["fp8"], dim)
    q = rng.integers(-2, 3, (new, 4, dim)).astype(np.float64)
    got, lse = hago.mx_attention(torch.from_numpy(q).to(TYPES[name]).to(DEV), cache, *on_gpu(table, lengths, offsets), scale=scale, lse=True)
    got, lse = got.double().cpu().numpy(), lse.double().cpu().numpy()
    seqs = ref.Sequences(table, lengths, offsets, pages, page)
    places = np.array([seqs.place(0, j) for j in range(length)])
    u = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}[name]
    for t in range(new):
        seen = places[:length - new + t + 1]
        for h in range(4):
            k, v = (r[seen[:, 0], h // 2, seen[:, 1]] for r in real)
            score = k @ q[t, h]
            best = (score if scale > 0 else -score).max()
            first = score == (best if scale > 0 else -best)
            want, size = v[first].mean(0), np.abs(v[first]).mean(0)
            limit = size * (2.0 ** -21 + 2 * first.sum() * 2.0 ** -24 + (2.0 ** -8 if name == "bf16" else 2.0 ** -16 if name == "f16" else 0)) + u * np.abs(want) + 2.0 ** -25
            assert (np.abs(got[t, h] - want) <= limit * (1 + u)).all(), (t, h)
            log = abs(scale) * best + np.log(first.sum())
            assert abs(lse[t, h] - log) <= 2.0 ** -21 * (abs(log) + 1), (t, h)


def test_scales_that_are_refused():
    """Beyond 2^100, and no numbers."""
    cache = hago.MXCache.empty(2, 1, 16, 64)
    where = on_gpu(np.zeros((1, 2), np.int32), np.array([4], np.int32), np.array([0, 4], np.int32))
    q = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device=DEV)
    for scale in (float("inf"), -float("inf"), float("nan"), 2.0 ** 101):
        with pytest.raises(hago.HagoError):
            hago.mx_attention(q, cache, *where, scale=scale)
