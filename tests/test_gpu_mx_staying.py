"""Workgroups of the microscaled products that go from tile to tile: from a last stage that computes (even numbers of stages of 256 k) as from
one that does not, between whole tiles, whose stores are counted, and ragged ones, and from one expert to another."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2103_14949_amd as hago
import test_gpu_mx as t
from oracle import mx_ref as mx

KERNELS = range(5)   # tiles through LDS; which of them stay depends on the format


@pytest.fixture
def kernels():
    def forced():
        for k in KERNELS:
            hago.set_test_hook(hago.HOOK_MX_KERNEL, k)
            yield k
    yield forced
    hago.set_test_hook(hago.HOOK_MX_KERNEL, -1)


def product(a, w):
    """Exact: sums that 64 bits hold."""
    return torch.from_numpy(a).to(t.DEV) @ torch.from_numpy(w).to(t.DEV).t().contiguous()


@pytest.mark.timeout(120)
@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("M,N,K", [(4096, 4096, 512), (2100, 4200, 512), (4096, 4096, 256), (1500, 6000, 1024), (3000, 4096, 2048), (4096, 3000, 768)])
def test_dense(kernels, M, N, K, fmt):
    rng = np.random.default_rng(M + K)
    a, w = t.operand(rng, M, K, fmt, True), t.operand(rng, N, K, "fp4", True)
    bias = torch.arange(N, dtype=torch.float32, device=t.DEV)
    da, dw = t.on_gpu(a, fmt, K), t.on_gpu(w, "fp4", K)
    exact = product(mx.decode(*a, fmt, K), mx.decode(*w, "fp4", K))
    want = {hago.F32: (exact + bias.double()).float(), hago.BF16: exact.to(torch.bfloat16), hago.F16: (exact + bias.double()).to(torch.float16)}
    for k in kernels():
        for out, b in ((hago.F32, bias), (hago.BF16, None), (hago.F16, bias)):
            assert torch.equal(hago.mx_dense(da, dw, b, out_dtype=out), want[out]), (k, out)


SIZES = [512, 300, 0, 1, 640, 129, 1024, 77, 256, 0, 384]   # 59 tiles of 64 rows, 31 of 128


@pytest.mark.timeout(120)
@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("N,K", [(2560, 512), (2500, 640), (2560, 1024), (2560, 256)])
def test_grouped(kernels, N, K, gather, fmt):
    rng = np.random.default_rng(N + K)
    a, w, off, index = t.group_case(rng, SIZES, N, K, fmt, gather, True, gap=3)
    bias = rng.integers(-50, 50, (len(SIZES), N)).astype(np.float32)
    av, wv = mx.decode(*a, fmt, K), mx.decode(*w, "fp4", K)
    av = av if index is None else av[index]
    args = (t.on_gpu(a, fmt, K), t.on_gpu(w, "fp4", K), torch.from_numpy(off).to(t.DEV), None if index is None else torch.from_numpy(index).to(t.DEV))
    exact = torch.full((len(av), N), 77.0, dtype=torch.float64, device=t.DEV)
    plain = exact.clone()
    for e in range(len(SIZES)):
        plain[off[e]:off[e + 1]] = product(av[off[e]:off[e + 1]], wv[e])
        exact[off[e]:off[e + 1]] = plain[off[e]:off[e + 1]] + torch.from_numpy(bias[e]).to(t.DEV).double()
    for k in kernels():
        for out, b, want in (("f32", bias, exact), ("bf16", bias, exact), ("bf16", None, plain)):
            result = torch.full((len(av), N), 77.0, dtype=t.TYPES[out], device=t.DEV)
            hago.mx_dense_grouped(*args, None if b is None else torch.from_numpy(b).to(t.DEV), out_dtype=t.OUT[out], out=result)
            assert torch.equal(result, want.to(t.TYPES[out])), (k, out)
