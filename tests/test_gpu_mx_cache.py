"""Writing a paged microscaled cache and reading it back, on the GPU against the oracle.  Codes of given numbers are exact, and so are their values up
to the one rounding to the type."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2103_14949_amd as hago
from cache_util import DEV, FORMATS, OUT, TYPES, layout, on_gpu
from oracle import cache_ref as ref


def filled(pages, heads, page, dim, k_fmt, v_fmt):
    """A cache of bytes that nobody wrote."""
    c = hago.MXCache.empty(pages, heads, page, dim, FORMATS[k_fmt], FORMATS[v_fmt])
    for t in (c.k_codes, c.k_scales, c.v_codes, c.v_scales):
        t.fill_(0xA5)
    return c


def same(got, want, dtype):
    want = torch.from_numpy(np.ascontiguousarray(want)).to(dtype)
    got = got.cpu()
    return torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(), want.nan_to_num())


def check_write(cache, k, v, seqs, k_fmt, v_fmt):
    """Every byte of the cache: the tokens' codes at their places, what it held before everywhere else."""
    dim = k.shape[2]
    for x, fmt, codes, scales in ((k, k_fmt, cache.k_codes, cache.k_scales), (v, v_fmt, cache.v_codes, cache.v_scales)):
        want_codes, want_scales = np.full(codes.shape, 0xA5, np.uint8), np.full(scales.shape, 0xA5, np.uint8)
        for t in range(x.shape[0]):
            row = seqs.row(t)
            place = row and seqs.place(*row)
            if place is None:
                continue
            c, s = ref.encode_row(x[t].double().numpy(), fmt)
            want_codes[place[0], :, place[1]], want_scales[place[0], :, place[1]] = c, s
        assert np.array_equal(codes.cpu().numpy(), want_codes) and np.array_equal(scales.cpu().numpy(), want_scales)


@pytest.mark.parametrize("k_fmt,v_fmt", [("fp8", "fp8"), ("fp8", "fp4"), ("fp4", "fp8"), ("fp4", "fp4")])
@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("new,lengths,heads,page,dim", [
    ([1], [1], 1, 1, 1), ([1], [700], 8, 64, 128), ([3, 0, 5], [3, 9, 40], 3, 7, 80), ([40], [33], 2, 16, 33), ([2, 1, 1, 9], [50, 1, 0, 4], 1, 48, 256),
    ([130, 7], [130, 64], 5, 64, 64), ([1, 1, 1, 1, 1], [5, 1, 64, 65, 3], 2, 64, 96)])
def test_write_and_read(new, lengths, heads, page, dim, name, k_fmt, v_fmt):
    """Lengths below the number of new tokens leave some before the sequence: they have no place."""
    table, lengths, offsets, pages = layout(new, lengths, page, seed=dim, rows_before=2)
    T = int(offsets[-1]) + 3
    seqs = ref.Sequences(table, lengths, offsets, pages, page)
    g = torch.Generator().manual_seed(page)
    k, v = ((torch.randn(T, heads, dim, generator=g) * torch.exp2(torch.randint(-20, 10, (T, heads, 1), generator=g))).to(TYPES[name]) for _ in range(2))
    cache = filled(pages, heads, page, dim, k_fmt, v_fmt)
    where = on_gpu(table, lengths, offsets)
    assert hago.mx_cache_write(cache, k.to(DEV), v.to(DEV), *where) is cache
    check_write(cache, k, v, seqs, k_fmt, v_fmt)
    # read back, into tensors whose other rows stay
    out = tuple(torch.full((T, heads, dim), 7.0, dtype=TYPES[name], device=DEV) for _ in range(2))
    assert hago.mx_cache_read(cache, *where, T, out_dtype=OUT[name], out=out) is not None
    values = hago.mx_cache_write(cache, k.to(DEV), v.to(DEV), *where, values=True)
    for x, fmt, got, simulated in ((k, k_fmt, out[0], values[0]), (v, v_fmt, out[1], values[1])):
        want = np.full((T, heads, dim), 7.0)
        for t in range(T):
            row = seqs.row(t)
            if row is None:
                continue
            value = ref.decode_row(*ref.encode_row(x[t].double().numpy(), fmt), fmt, dim)
            assert same(simulated[t], value, TYPES[name])
            if seqs.place(*row) is not None:
                want[t] = value
        assert same(got, want, TYPES[name])


@pytest.mark.parametrize("name,offset", [("bf16", 0), ("f16", 1), ("f32", 1), ("bf16", 3)])
def test_strides(name, offset):
    """Keys and values inside the result of one product, and heads first; addresses off 16 bytes."""
    table, lengths, offsets, pages = layout([13, 4], [20, 4], 5)
    seqs = ref.Sequences(table, lengths, offsets, pages, 5)
    g = torch.Generator().manual_seed(1)
    qkv = torch.randn(17, 9, 44, generator=g).to(TYPES[name])
    dev = torch.empty(qkv.numel() + offset, dtype=qkv.dtype, device=DEV)[offset:].view(qkv.shape)
    dev.copy_(qkv)
    where = on_gpu(table, lengths, offsets)
    cache = filled(pages, 2, 5, 44, "fp8", "fp4")
    hago.mx_cache_write(cache, dev[:, 5:7], dev[:, 7:9], *where)
    check_write(cache, qkv[:, 5:7], qkv[:, 7:9], seqs, "fp8", "fp4")
    cache = filled(pages, 2, 5, 44, "fp8", "fp4")
    hago.mx_cache_write(cache, dev[:, 5:7].transpose(0, 1).contiguous().transpose(0, 1), dev[:, 7:8].expand(17, 2, 44), *where)
    check_write(cache, qkv[:, 5:7], qkv[:, 7:8].expand(17, 2, 44), seqs, "fp8", "fp4")


def test_a_table_with_rows_apart():
    table, lengths, offsets, pages = layout([3, 3], [9, 12], 4)
    wide = np.full((2, table.shape[1] + 5), 10 ** 6, np.int32)
    wide[:, :table.shape[1]] = table
    k = torch.randn(6, 1, 32, generator=torch.Generator().manual_seed(1))
    cache = filled(pages, 1, 4, 32, "fp8", "fp8")
    t, n, o = on_gpu(wide, lengths, offsets)
    hago.mx_cache_write(cache, k.to(DEV), k.to(DEV), t[:, :table.shape[1]], n, o)
    check_write(cache, k, k, ref.Sequences(table, lengths, offsets, pages, 4), "fp8", "fp8")


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_numbers_that_are_none(fmt):
    """A block with an infinity or NaN stands for NaN; others of its row do not."""
    x = torch.randn(4, 1, 96, generator=torch.Generator().manual_seed(1))
    x[0, 0, 5], x[1, 0, 40], x[2, 0, 95] = float("nan"), float("inf"), -float("inf")
    x[3] = 0
    table, lengths, offsets, pages = layout([4], [4], 4)
    where = on_gpu(table, lengths, offsets)
    cache = filled(pages, 1, 4, 96, fmt, fmt)
    values = hago.mx_cache_write(cache, x.to(DEV), x.to(DEV), *where, values=True)
    check_write(cache, x, x, ref.Sequences(table, lengths, offsets, pages, 4), fmt, fmt)
    got = hago.mx_cache_read(cache, *where, 4, out_dtype=hago.F32)
    for a, b in zip(values, got):
        assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(), b.nan_to_num())
        assert a.isnan().view(4, 3, 32).all(-1).tolist() == [[True, False, False], [False, True, False], [False, False, True], [False] * 3]


def test_places_that_are_none_and_offsets_that_break_the_contract():
    """Entries of the table that are no page, and lengths beyond the table: nothing is written there.  Offsets out of range: nothing out of range."""
    table = np.array([[1, -1, 5, 2], [0, 3, 2 ** 31 - 1, -2 ** 31]], np.int32)
    k = torch.randn(20, 1, 32, generator=torch.Generator().manual_seed(1))
    for lengths, offsets in (([19, 16], [0, 12, 20]), ([2 ** 31 - 1, 3], [0, 12, 20]), ([-5, -2 ** 31], [0, 12, 20])):
        seqs = ref.Sequences(table, lengths, offsets, 4, 4)
        cache = filled(4, 1, 4, 32, "fp8", "fp4")
        hago.mx_cache_write(cache, k.to(DEV), k.to(DEV), *on_gpu(table, np.array(lengths, np.int32), np.array(offsets, np.int32)))
        check_write(cache, k, k, seqs, "fp8", "fp4")
    for offsets in ([5, 3, 1], [-7, 2 ** 31 - 1, 4], [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1]):
        where = on_gpu(table, np.array([9, 9], np.int32), np.array(offsets, np.int32))
        hago.mx_cache_write(filled(4, 1, 4, 32, "fp8", "fp4"), k.to(DEV), k.to(DEV), *where)
        hago.mx_cache_read(filled(4, 1, 4, 32, "fp8", "fp4"), *where, 20)
    torch.cuda.synchronize()


def test_nothing_to_do():
    cache = hago.MXCache.empty(2, 1, 4, 32)
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)  # noqa: E731
    hago.mx_cache_write(cache, torch.zeros(0, 1, 32, device=DEV), torch.zeros(0, 1, 32, device=DEV), i(1, 2), i(1), i(2))
    hago.mx_cache_write(cache, torch.zeros(3, 1, 32, device=DEV), torch.zeros(3, 1, 32, device=DEV), i(0, 2), i(0), i(1))
    empty = hago.MXCache.empty(0, 1, 4, 32)
    hago.mx_cache_write(empty, torch.zeros(3, 1, 32, device=DEV), torch.zeros(3, 1, 32, device=DEV), i(1, 2), i(1) + 3, torch.tensor([0, 3], dtype=torch.int32, device=DEV))
    assert hago.mx_cache_read(cache, i(0, 2), i(0), i(1), 0)[0].shape == (0, 1, 32)
    torch.cuda.synchronize()


@pytest.mark.parametrize("seqs", [1, 63, 64, 65, 700])
def test_many_sequences(seqs):
    """Rows find their sequence however many there are, empty ones among them."""
    rng = np.random.default_rng(seqs)
    new = rng.integers(0, 4, seqs)
    new[rng.integers(0, seqs)] = 3
    lengths = new + rng.integers(0, 9, seqs)
    table, lengths, offsets, pages = layout(list(new), list(lengths), 4, seed=seqs)
    k = torch.randn(int(offsets[-1]), 1, 32, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    cache = filled(pages, 1, 4, 32, "fp8", "fp8")
    hago.mx_cache_write(cache, k.to(DEV), k.to(DEV), *on_gpu(table, lengths, offsets))
    check_write(cache, k, k, ref.Sequences(table, lengths, offsets, pages, 4), "fp8", "fp8")


def test_beyond_32_bits():
    """Pages whose bytes begin behind 2^31 and 2^32."""
    pages, page, heads = 70000, 64, 8   # 4.6 GB of codes a tensor at 128 columns
    cache = hago.MXCache.empty(pages, heads, page, 128)
    table = np.array([[pages - 1, 33000, 65600, 5]], np.int32)
    k, v = (torch.randn(200, heads, 128, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16) for i in range(2))
    where = on_gpu(table, np.array([200], np.int32), np.array([0, 200], np.int32))
    values = hago.mx_cache_write(cache, k.to(DEV), v.to(DEV), *where, values=True)
    got = hago.mx_cache_read(cache, *where, 200)
    assert torch.equal(got[0], values[0]) and torch.equal(got[1], values[1])
    codes, scales = ref.encode_row(k[70].double().numpy(), "fp8")
    assert np.array_equal(cache.k_codes[33000, :, 6].cpu().numpy(), codes) and np.array_equal(cache.k_scales[33000, :, 6].cpu().numpy(), scales)


def test_prepared_calls_and_graphs():
    """A prepared write holds its cache's tensors; a captured write and read, replayed with other tokens, lengths and tables."""
    table, lengths, offsets, pages = layout([2, 3], [9, 5], 4)
    where = on_gpu(table, lengths, offsets)
    k, v = (torch.randn(5, 2, 64, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    cache = filled(pages, 2, 4, 64, "fp8", "fp4")
    for t in (cache.k_codes, cache.v_codes):
        t.zero_()
    call = hago.mx_cache_write(cache, k, v, *where, prepare=True)
    assert call() is cache
    out = hago.mx_cache_read(cache, *where, 5)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        hago.mx_cache_write(cache, k, v, *where)
        hago.mx_cache_read(cache, *where, 5, out=out)
    for turn in range(3):
        k.normal_()
        v.normal_()
        where[1].add_(1)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], hago.mx_quantize(k.view(-1, 64), hago.MX_FP8, values=True)[1].view_as(k))
        assert torch.equal(out[1], hago.mx_quantize(v.view(-1, 64), hago.MX_FP4, values=True)[1].view_as(v))
