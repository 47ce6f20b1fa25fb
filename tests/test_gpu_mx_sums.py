"""Sums of 8-bit rows.  32-bit results: every term counts, however far below the others it lies.  16-bit results: what the matrix instruction cuts off.

The terms of the first tests are multiples of 2^-10 and sum to less than 2^13 in size, so binary32 holds every partial sum and the result is
exact, though each row has codes of 2^-9 beside ones of 448."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2103_14949_amd as hago
import test_gpu_mx as t
from oracle import mx_ref as mx

KERNELS = range(13)


@pytest.fixture
def kernels():
    def forced():
        for k in KERNELS:
            hago.set_test_hook(hago.HOOK_MX_KERNEL, k)
            yield k
    yield forced
    hago.set_test_hook(hago.HOOK_MX_KERNEL, -1)


def rows_of_far_codes(rng, rows, K):
    """Codes below 2^-2 of either sign, and in every row one of 128 to 448 (three up to 300 columns)."""
    codes = rng.integers(0, 0x28, (rows, mx.padded(K))) | rng.integers(0, 2, (rows, mx.padded(K))) << 7
    for row in codes:
        at = rng.choice(K, min(K, 3 if K <= 300 else 1), replace=False)
        row[at] = rng.integers(0x70, 0x7F, len(at)) | rng.integers(0, 2, len(at)) << 7
    codes[:, K:] = 0
    scales = np.full((rows, mx.padded(K) // 32), 127, np.uint8)
    scales[:, -(-K // 32):] = 0
    return mx.pack(codes, "fp8"), scales


def weights(rng, lead, N, K):
    codes = rng.integers(0, 16, (*lead, N, mx.padded(K)))
    codes[..., K:] = 0
    scales = np.full((*lead, N, mx.padded(K) // 32), 127, np.uint8)
    scales[..., -(-K // 32):] = 0
    return mx.pack(codes, "fp4"), scales


@pytest.mark.parametrize("M,N,K", [(1, 16, 33), (17, 48, 64), (5, 130, 128), (64, 100, 300), (130, 257, 1024), (300, 520, 2048)])
def test_dense(kernels, M, N, K):
    rng = np.random.default_rng(M + N + K)
    a, w = rows_of_far_codes(rng, M, K), weights(rng, (), N, K)
    av, wv = mx.decode(*a, "fp8", K), mx.decode(*w, "fp4", K)
    assert (np.abs(av) @ np.abs(wv).T).max() < 2 ** 13
    bias = rng.integers(-9, 10, N).astype(np.float32)
    da, dw, db = t.on_gpu(a, "fp8", K), t.on_gpu(w, "fp4", K), torch.from_numpy(bias).to(t.DEV)
    for k in kernels():
        assert t.same_values(hago.mx_dense(da, dw, db, out_dtype=hago.F32), av @ wv.T + bias, torch.float32), k


@pytest.mark.parametrize("gather", [False, True])
def test_grouped(kernels, gather):
    rng = np.random.default_rng(4)
    sizes, N, K = [40, 0, 3, 200, 17, 1], 150, 384
    off = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    T = int(off[-1])
    a, w = rows_of_far_codes(rng, T, K), weights(rng, (len(sizes),), N, K)
    index = rng.integers(0, T, T).astype(np.int32) if gather else None
    av, wv = mx.decode(*a, "fp8", K), mx.decode(*w, "fp4", K)
    av = av if index is None else av[index]
    want = np.concatenate([av[off[e]:off[e + 1]] @ wv[e].T for e in range(len(sizes))])
    args = (t.on_gpu(a, "fp8", K), t.on_gpu(w, "fp4", K), torch.from_numpy(off).to(t.DEV), None if index is None else torch.from_numpy(index).to(t.DEV))
    for k in kernels():
        assert t.same_values(hago.mx_dense_grouped(*args, out_dtype=hago.F32), want, torch.float32), k


@pytest.mark.parametrize("K", [64, 128, 192, 1000])
def test_normal_rows(kernels, K):
    """The two parts of every 16 k are added to the running sum one after the other, each at the cost of 2^-23 of it at most."""
    rng = np.random.default_rng(K)
    M, N = 70, 300
    a, w = t.operand(rng, M, K, "fp8"), t.operand(rng, N, K, "fp4")
    av, wv = mx.decode(*a, "fp8", K), mx.decode(*w, "fp4", K)
    want, terms = av @ wv.T, np.abs(av) @ np.abs(wv).T
    bound = (2 * -(-K // 16) + 2) * 2.0 ** -23 * terms
    da, dw = t.on_gpu(a, "fp8", K), t.on_gpu(w, "fp4", K)
    for k in kernels():
        assert (np.abs(t.wide(hago.mx_dense(da, dw, out_dtype=hago.F32)) - want) <= bound).all(), k


def cut_at_most(a, w, K):
    """By the description of the instruction (include/hago.h), how much of a sum it may cut off: of every 16 k, less than 2^(E - 13) of each product
    but the largest; E from the exponents of codes that are not zero (a subnormal code has the least exponent)."""
    ac, wc = mx.unpack(a[0], "fp8")[:, :K].astype(int), mx.unpack(w[0], "fp4")[:, :K].astype(int)
    none = -10 ** 6
    ea = np.where(ac & 127, np.maximum(ac >> 3 & 15, 1) - 7, none) + np.repeat(a[1].astype(int) - 127, 32, -1)[:, :K]
    ew = np.where(wc & 7, np.maximum(wc >> 1 & 3, 1) - 1, none) + np.repeat(w[1].astype(int) - 127, 32, -1)[:, :K]
    total = np.zeros((len(ac), len(wc)))
    for first in range(0, K, 32):
        for half in (0, 8):
            k = [c for c in range(first + half, min(first + half + 24, K)) if (c - first - half) % 16 < 8]
            if not k:
                continue
            e = np.maximum.reduce([ea[:, c, None] + ew[None, :, c] for c in k])
            total += np.where(e > none // 2, 15 * np.exp2(np.maximum(e, -500) - 13.0), 0)
    return total


@pytest.mark.parametrize("far", [False, True])
@pytest.mark.parametrize("K", [64, 100, 384])
def test_16_bit_results(kernels, K, far):
    rng = np.random.default_rng(K + 1)
    M, N = 40, 90
    a, w = (rows_of_far_codes(rng, M, K), weights(rng, (), N, K)) if far else (t.operand(rng, M, K, "fp8"), t.operand(rng, N, K, "fp4"))
    av, wv = mx.decode(*a, "fp8", K), mx.decode(*w, "fp4", K)
    want, terms = av @ wv.T, np.abs(av) @ np.abs(wv).T
    da, dw = t.on_gpu(a, "fp8", K), t.on_gpu(w, "fp4", K)
    cut = cut_at_most(a, w, K) + (-(-K // 16) + 2) * 2.0 ** -23 * terms
    for out, half_unit, least in (("bf16", 2.0 ** -8, 0), ("f16", 2.0 ** -11, 2.0 ** -25)):   # (as in product_bound)
        for k in kernels():
            got = t.wide(hago.mx_dense(da, dw, out_dtype=t.OUT[out]))
            assert (np.abs(got - want) <= cut + half_unit * (np.abs(want) + cut) + least).all(), (k, out)
