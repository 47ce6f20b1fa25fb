"""Attention over a paged microscaled cache where sequences have many rows, whose kernel is another: chunks and prompts, in every form; and both kernels on a cache
beyond 2^32 bytes."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2103_14949_amd as hago
from cache_util import DEV, check_attention, layout, on_gpu, random_cache
from oracle import cache_ref as ref
from test_gpu_mx_attention import run


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("k_fmt,v_fmt", [("fp8", "fp8"), ("fp8", "fp4"), ("fp4", "fp8"), ("fp4", "fp4")])
@pytest.mark.parametrize("dim", [3, 32, 50, 64, 72, 96, 128, 200, 256])
def test_formats_and_columns(dim, k_fmt, v_fmt, name):
    run([90, 1, 0, 41], [130, 77, 5, 41], 4, 2, dim, 16, k_fmt, v_fmt, name, seed=dim)


@pytest.mark.parametrize("page", [1, 7, 8, 16, 40, 64, 128, 500])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 1), (True, 70), (False, 0), (False, 33), (True, 10 ** 6)])
def test_pages_and_windows(page, causal, window):
    run([150, 3, 90], [290, 200, 90], 2, 1, 64, page, "fp8", "fp4", causal=causal, window=window, seed=page)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("length", [63, 64, 65, 127, 128, 129, 192, 193, 256, 257, 320, 449])
def test_lengths(length, dim):
    """Tiles of 64 keys and of 256 (128) rows, one more and one less."""
    run([length], [length], 1, 1, dim, 32, seed=length)
    run([64], [length + 100], 4, 1, dim, 32, seed=length)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (6, 2), (16, 1), (17, 1)])
def test_heads(heads, kv_heads):
    run([70, 20], [170, 20], heads, kv_heads, 64, 64, seed=heads)


@pytest.mark.parametrize("window", [0, 5])
def test_rows_that_see_nothing(window):
    """Chunks longer than their sequences: the rows that stand before them see nothing."""
    run([200, 90, 100], [70, 0, -3], 2, 1, 64, 8, window=window, seed=1)
    run([200, 90, 100], [70, 0, -3], 2, 1, 64, 8, window=window, causal=False, seed=1)


@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0, 1e-30])
def test_scales(scale):
    run([100], [140], 2, 1, 64, 16, name="f16", scale=scale, seed=2)
    run([100], [140], 2, 1, 64, 16, name="bf16", scale=scale, seed=2)


def test_long_chunks_are_cut_and_joined():
    run([70], [6000], 2, 1, 64, 64, "fp4", "fp8", seed=3)
    run([65, 64], [3000, 900], 2, 1, 128, 64, name="f16", seed=4)
    run([70], [6000], 2, 1, 64, 64, window=2500, seed=5)
    run([3], [6000], 2, 1, 64, 64, window=2500, causal=False, seed=6)


def test_many_sequences():
    """More sequences than a wavefront has lanes, some without rows."""
    rng = np.random.default_rng(11)
    new = rng.integers(0, 3, 70) * rng.integers(30, 60, 70)
    run(list(new), list(new + rng.integers(0, 40, 70)), 4, 1, 32, 16, seed=7)


def test_large_scores_raise_the_maximum():
    """Scores that grow along the keys by far more than the kernel lets them pass, and in the last tile alone."""
    rng = np.random.default_rng(5)
    table, lengths, offsets, pages = layout([96], [400], 16)
    cache, keys, values = random_cache(rng, pages, 1, 16, 64, "fp8", "fp8")
    seqs = ref.Sequences(table, lengths, offsets, pages, 16)
    for j in range(400):   # every scale byte of a key up by a binary order each 50 positions, and by six in the last ten
        p, at = seqs.place(0, j)
        up = j // 50 + (6 if j >= 390 else 0)
        cache.k_scales[p, 0, at] += up
        keys[p, 0, at] *= 2.0 ** up
    q = torch.from_numpy(rng.standard_normal((96, 2, 64))).to(torch.bfloat16)
    out, lse = hago.mx_attention(q.to(DEV), cache, *on_gpu(table, lengths, offsets), lse=True)
    check_attention(out, "bf16", q.double().numpy(), keys, values, seqs, 0.125, lse=lse)


def test_pages_that_are_gone():
    rng = np.random.default_rng(7)
    for page in (16, 5):
        table, lengths, offsets, pages = layout([70, 66], [320, 90], page)
        cache, keys, values = random_cache(rng, pages, 2, page, 64, "fp8", "fp4")
        table[0, :3] = [-1, pages, 2 ** 31 - 1]
        table[0, 9], table[1, 2] = -5, -2 ** 31
        q = torch.from_numpy(rng.standard_normal((136, 4, 64))).to(torch.bfloat16)
        out = hago.mx_attention(q.to(DEV), cache, *on_gpu(table, lengths, offsets))
        check_attention(out, "bf16", q.double().numpy(), keys, values, ref.Sequences(table, lengths, offsets, pages, page), 0.125)
        table[:] = -1
        out, lse = hago.mx_attention(q.to(DEV), cache, *on_gpu(table, lengths, offsets), lse=True)
        assert (out == 0).all() and lse.isneginf().all()


def test_offsets_that_break_the_contract():
    rng = np.random.default_rng(8)
    cache, _, _ = random_cache(rng, 6, 1, 16, 64, "fp8", "fp8")
    q = torch.randn(200, 2, 64, device=DEV, dtype=torch.bfloat16)
    table = np.arange(6, dtype=np.int32).reshape(2, 3)
    for offsets in ([50, 30, 10], [-7, 2 ** 31 - 1, 4], [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1], [0, 200, -200], [-2 ** 31, 200, 200], [0, 200, 200]):
        for lengths in ([40, 40], [2 ** 31 - 1, -2 ** 31]):
            hago.mx_attention(q, cache, *on_gpu(table, np.array(lengths, np.int32), np.array(offsets, np.int32)))
    torch.cuda.synchronize()


def test_the_same_twice_and_in_a_graph():
    """No result depends on the order in which workgroups come: bit by bit the same, eager and replayed."""
    rng = np.random.default_rng(9)
    table, lengths, offsets, pages = layout([100, 1, 300], [3000, 700, 300], 16)
    cache, _, _ = random_cache(rng, pages, 2, 16, 128, "fp8", "fp4")
    where = on_gpu(table, lengths, offsets)
    q = torch.randn(401, 8, 128, device=DEV, dtype=torch.bfloat16)
    want = hago.mx_attention(q, cache, *where)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = hago.mx_attention(q, cache, *where)
    for _ in range(3):
        assert torch.equal(hago.mx_attention(q, cache, *where), want)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("new", [1, 130])
@pytest.mark.parametrize("page", [64, 60])
def test_beyond_32_bits(new, page):
    """Pages whose codes begin behind 2^31 and 2^32: the same as in a small cache that holds the same rows."""
    pages, heads, total = 70000, 8, 300
    table = np.array([[pages - 1, 33000, 65600, 5, 69000]], np.int32)
    k, v = (torch.randn(total, heads, 128, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16).to(DEV) for i in range(2))
    q = torch.randn(new, 2 * heads, 128, device=DEV, dtype=torch.bfloat16)
    outs = []
    for n, t in ((pages, table), (5, np.arange(5, dtype=np.int32)[None])):
        cache = hago.MXCache.empty(n, heads, page, 128)
        where = on_gpu(t, np.array([total], np.int32))
        hago.mx_cache_write(cache, k, v, *where, *on_gpu(np.array([0, total], np.int32)))
        outs.append(hago.mx_attention(q, cache, *where, *on_gpu(np.array([0, new], np.int32))))
    assert torch.equal(*outs) and outs[0].isfinite().all()


@pytest.mark.parametrize("most", [2, 60])
@pytest.mark.parametrize("seqs", [257, 1024, 1025, 3000])
def test_a_plan_of_many_sequences(seqs, most):
    """More sequences than every workgroup looks at: the same as in calls of a hundred, bit by bit where none is cut."""
    rng = np.random.default_rng(seqs)
    new = rng.integers(0, most, seqs)
    lengths = np.minimum(new + rng.integers(0, 9, seqs), 64)
    table, lengths, offsets, pages = layout(list(new), list(lengths), 16, seed=seqs)
    cache, _, _ = random_cache(rng, pages, 2, 16, 64, "fp8", "fp4")
    q = torch.randn(int(offsets[-1]), 4, 64, device=DEV, dtype=torch.bfloat16)
    got, lse = hago.mx_attention(q, cache, *on_gpu(table, lengths, offsets), lse=True)
    for first in range(0, seqs, 100):
        end = min(first + 100, seqs)
        a, b = int(offsets[first]), int(offsets[end])
        part = hago.mx_attention(q[a:b], cache, *on_gpu(table[first:end], lengths[first:end], offsets[first:end + 1] - a), lse=True)
        assert torch.equal(got[a:b], part[0]) and torch.equal(lse[a:b], part[1])


def test_a_plan_with_long_sequences():
    """Some of many are cut."""
    new, lengths = [1] * 300, [3] * 300
    lengths[7], lengths[299] = 30000, 9000
    run(new, lengths, 2, 1, 32, 64, seed=13)
    offsets = [[0, 300, 5], [-3, 2 ** 31 - 1]]   # and offsets that break the contract, with as many
    cache = hago.MXCache.empty(8, 1, 16, 32)
    q = torch.randn(400, 2, 32, device=DEV, dtype=torch.bfloat16)
    for bad in offsets:
        off = np.resize(np.array(bad, np.int32), 301)
        hago.mx_attention(q, cache, *on_gpu(np.zeros((300, 2), np.int32), np.full(300, 30, np.int32), off))
    torch.cuda.synchronize()
