"""What the microscaled operators refuse, on the host and before anything is launched: by the C ABI's statuses and by the binding."""
import math
import os

import numpy as np
import pytest
import torch

import paper_2103_14949_amd as hago


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(hago.library_path()):
        from paper_2103_14949_amd import build
        build.build()
    return hago.lib()


P = 0x1000   # an aligned pointer that is never followed
NULL, SHAPE, DTYPE, PARAM = 1, 2, 3, 5


@pytest.mark.parametrize("name,wide", [("hago_mx_quantize", 1), ("hago_mx_silu_mul", 2)])
def test_quantize_and_silu_mul(L, name, wide):
    def call(x=P, t=hago.BF16, rows=4, cols=64, stride=None, fmt=hago.MX_FP4, codes=P, scales=P, values=P):
        return getattr(L, name)(x, t, rows, cols, wide * cols if stride is None else stride, fmt, codes, scales, values, None)
    assert call(x=None) == NULL and call(codes=None) == NULL and call(scales=None) == NULL
    assert call(rows=-1) == SHAPE and call(cols=-1, stride=64) == SHAPE and call(stride=wide * 64 - 1) == SHAPE
    assert call(cols=2 ** 31 - 128, stride=2 ** 33) == SHAPE and call(rows=2 ** 40, stride=2 ** 40) == SHAPE
    assert call(cols=2 ** 62, stride=2 ** 62) == SHAPE
    for t in (hago.U8, hago.I8, hago.I16, hago.I32, hago.I24, 8, -1):
        assert call(t=t) == DTYPE
    assert call(fmt=2) == PARAM and call(fmt=-1) == PARAM
    assert call(x=P + 1) == PARAM and call(values=P + 1) == PARAM and call(codes=P + 8) == PARAM and call(scales=P + 2) == PARAM
    assert call(t=hago.F32, x=P + 2) == PARAM
    assert call(rows=0, x=None, codes=None, scales=None, values=None) == 0 and call(cols=0, stride=0, x=None, codes=None, scales=None) == 0
    assert call(rows=0, t=hago.U8) == DTYPE   # (also of empty tensors)


def test_rmsnorm(L):
    def call(x=P, res=P, gamma=P, t=hago.BF16, rows=4, cols=64, stride=64, eps=1e-5, fmt=hago.MX_FP8, res_out=2 * P, codes=P, scales=P, values=None):
        return L.hago_mx_rmsnorm(x, res, gamma, t, rows, cols, stride, eps, fmt, res_out, codes, scales, values, None)
    assert call(x=None) == NULL and call(codes=None) == NULL and call(scales=None) == NULL
    assert call(rows=-1) == SHAPE and call(stride=63) == SHAPE
    assert call(t=hago.I8) == DTYPE
    for eps in (-1e-9, math.inf, math.nan):
        assert call(eps=eps) == PARAM
    assert call(res=P + 1) == PARAM and call(gamma=P + 1) == PARAM and call(res_out=P + 1) == PARAM
    assert call(res_out=P, stride=65) == PARAM   # in place of x with rows at another distance
    assert call(rows=0, x=None, codes=None, scales=None) == 0


def test_products(L):
    def dense(a=P, s=P, f=hago.MX_FP8, w=P, ws=P, b=None, M=4, N=8, K=64, t=hago.BF16, out=P):
        return L.hago_mx_dense(a, s, f, w, ws, b, M, N, K, t, out, None)

    def grouped(a=P, s=P, f=hago.MX_FP8, rows=4, index=None, w=P, ws=P, b=None, off=P, T=4, E=3, N=8, K=64, t=hago.BF16, out=P):
        return L.hago_mx_dense_grouped(a, s, f, rows, index, w, ws, b, off, T, E, N, K, t, out, None)
    for call in (dense, grouped):
        for name in ("a", "s", "w", "ws", "out"):
            assert call(**{name: None}) == NULL, name
        assert call(N=-1) == SHAPE and call(K=-1) == SHAPE and call(K=2 ** 22 + 1) == SHAPE and call(N=2 ** 31) == SHAPE
        for t in (hago.I8, hago.I32, 8):
            assert call(t=t) == DTYPE
        assert call(f=2) == PARAM
        for name, off in (("a", 8), ("w", 8), ("s", 2), ("ws", 1), ("b", 2), ("out", 1)):
            assert call(**{name: P + off}) == PARAM, name
        assert call(t=hago.F32, out=P + 2) == PARAM
        assert call(N=0, out=None) == 0
    assert dense(M=-1) == SHAPE and dense(M=2 ** 31 - 300, N=2 ** 31 - 300) == SHAPE and dense(M=0, a=None, out=None) == 0
    assert grouped(off=None) == NULL and grouped(off=P + 2) == PARAM and grouped(index=P + 2) == PARAM
    assert grouped(T=-1) == SHAPE and grouped(E=-1) == SHAPE and grouped(rows=0) == SHAPE
    assert grouped(rows=3) == SHAPE and grouped(rows=3, index=P, K=2 ** 22 + 1) == SHAPE   # fewer rows than results, without an index
    assert grouped(rows=2 ** 24, index=P, K=128) == SHAPE   # indexed activations of 2^31 bytes
    assert grouped(T=0, out=None) == 0 and grouped(E=0) == 0


def MX(rows, cols, fmt, lead=()):
    wide = (cols + 127) // 128 * 128
    z = lambda n: torch.zeros(*lead, rows, n, dtype=torch.uint8)  # noqa: E731
    return hago.MX(z(wide // 2 if fmt == hago.MX_FP4 else wide), z(wide // 32), fmt, cols)


X = torch.zeros(4, 64, dtype=torch.bfloat16)
A, W, WG = MX(4, 64, hago.MX_FP8), MX(8, 64, hago.MX_FP4), MX(8, 64, hago.MX_FP4, (3,))
OFF = torch.zeros(4, dtype=torch.int32)


@pytest.mark.parametrize("call,error", [
    (lambda: hago.mx_quantize(np.zeros((4, 64), np.float32), hago.MX_FP4), TypeError),
    (lambda: hago.mx_quantize(X.double(), hago.MX_FP4), TypeError),
    (lambda: hago.mx_quantize(X[0], hago.MX_FP4), AssertionError),
    (lambda: hago.mx_quantize(X.t(), hago.MX_FP4), AssertionError),
    (lambda: hago.mx_quantize(X.expand(2, 4, 64)[0].as_strided((4, 64), (0, 1)), hago.MX_FP4), AssertionError),
    (lambda: hago.mx_quantize(X, 2), AssertionError),
    (lambda: hago.mx_quantize(X, "fp4"), TypeError),
    (lambda: hago.mx_quantize(X, hago.MX_FP4, out=MX(4, 64, hago.MX_FP8)), AssertionError),
    (lambda: hago.mx_quantize(X, hago.MX_FP4, out=MX(3, 64, hago.MX_FP4)), AssertionError),
    (lambda: hago.mx_quantize(X, hago.MX_FP4, values=torch.zeros(4, 64)), AssertionError),
    (lambda: hago.mx_quantize(X, hago.MX_FP4), AssertionError),   # a host tensor
    (lambda: hago.mx_silu_mul(X[:, :63], hago.MX_FP4), AssertionError),
    (lambda: hago.mx_rmsnorm(X, gamma=torch.zeros(64)), AssertionError),
    (lambda: hago.mx_rmsnorm(X, gamma=torch.zeros(63, dtype=torch.bfloat16)), AssertionError),
    (lambda: hago.mx_rmsnorm(X, residual=X[:3]), AssertionError),
    (lambda: hago.mx_rmsnorm(X, residual=X, out_residual=X.float()), AssertionError),
    (lambda: hago.mx_rmsnorm(X, eps="x"), TypeError),
    (lambda: hago.mx_dense(A, MX(8, 64, hago.MX_FP8)), AssertionError),
    (lambda: hago.mx_dense(A, MX(8, 65, hago.MX_FP4)), AssertionError),
    (lambda: hago.mx_dense(A, WG), AssertionError),
    (lambda: hago.mx_dense(hago.MX(A.codes, A.scales, hago.MX_FP4, 64), W), AssertionError),
    (lambda: hago.mx_dense(hago.MX(A.codes, A.scales[:3], A.fmt, 64), W), AssertionError),
    (lambda: hago.mx_dense(hago.MX(A.codes, A.scales.float(), A.fmt, 64), W), AssertionError),
    (lambda: hago.mx_dense(A, W, torch.zeros(7)), AssertionError),
    (lambda: hago.mx_dense(A, W, torch.zeros(8, dtype=torch.bfloat16)), AssertionError),
    (lambda: hago.mx_dense(A, W, out=torch.zeros(4, 8)), AssertionError),
    (lambda: hago.mx_dense(A, W, out_dtype=77), KeyError),
    (lambda: hago.mx_dense(A, W), AssertionError),
    (lambda: hago.mx_dense_grouped(A, W, OFF), AssertionError),
    (lambda: hago.mx_dense_grouped(A, WG, None), TypeError),
    (lambda: hago.mx_dense_grouped(A, WG, OFF[:3]), AssertionError),
    (lambda: hago.mx_dense_grouped(A, WG, OFF.long()), AssertionError),
    (lambda: hago.mx_dense_grouped(A, WG, OFF, rows=torch.zeros(5)), AssertionError),
    (lambda: hago.mx_dense_grouped(A, WG, OFF, bias=torch.zeros(8)), AssertionError),
    (lambda: hago.mx_dense_grouped(A, WG, OFF), AssertionError),
])
def test_the_binding_refuses(L, call, error):
    with pytest.raises(error):
        call()
