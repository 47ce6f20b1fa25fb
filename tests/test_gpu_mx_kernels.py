"""Every kernel of the microscaled products, forced in turn, at sizes inside, at and across its tiles."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2103_14949_amd as hago
import test_gpu_mx as t
from oracle import mx_ref as mx

KERNELS = range(13)   # 0 to 4: tiles through LDS; 5 on: few rows


@pytest.fixture
def kernels():
    """The kernels, each forced while it is the current one."""
    def forced():
        for k in KERNELS:
            hago.set_test_hook(hago.HOOK_MX_KERNEL, k)
            yield k
    yield forced
    hago.set_test_hook(hago.HOOK_MX_KERNEL, -1)


@pytest.mark.parametrize("M,N,K", t.SIZES)
@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_dense(kernels, M, N, K, fmt):
    rng = np.random.default_rng(M + N + K)
    bias = rng.standard_normal(N).astype(np.float32)
    for exact in (True, False):
        a, w = t.operand(rng, M, K, fmt, exact), t.operand(rng, N, K, "fp4", exact)
        av, wv = mx.decode(*a, fmt, K), mx.decode(*w, "fp4", K)
        want, terms = av @ wv.T, np.abs(av) @ np.abs(wv).T
        da, dw, db = t.on_gpu(a, fmt, K), t.on_gpu(w, "fp4", K), torch.from_numpy(bias).to(t.DEV)
        for k in kernels():
            if exact:
                for out in ("f32", "f16"):
                    assert t.same_values(hago.mx_dense(da, dw, out_dtype=t.OUT[out]), want, t.TYPES[out]), (k, out)
            else:
                got = t.wide(hago.mx_dense(da, dw, db))
                assert (np.abs(got - (want + bias)) <= t.product_bound(terms + np.abs(bias), want + bias, K, fmt, "bf16")).all(), k


@pytest.mark.parametrize("sizes,N,K", t.GROUPS)
@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("gather", [False, True])
def test_grouped(kernels, sizes, N, K, fmt, gather):
    rng = np.random.default_rng(sum(sizes) + N + K)
    gap = 3   # rows in no group at either end
    a, w, off, index = t.group_case(rng, sizes, N, K, fmt, gather, True, gap)
    av, wv = mx.decode(*a, fmt, K), mx.decode(*w, "fp4", K)
    av = av if index is None else av[index]
    want = np.full((len(av), N), 77.0)
    for e in range(len(sizes)):
        want[off[e]:off[e + 1]] = av[off[e]:off[e + 1]] @ wv[e].T
    args = (t.on_gpu(a, fmt, K), t.on_gpu(w, "fp4", K), torch.from_numpy(off).to(t.DEV), None if index is None else torch.from_numpy(index).to(t.DEV))
    for out in ("f32", "bf16"):
        for k in kernels():
            result = torch.full((len(av), N), 77.0, dtype=t.TYPES[out], device=t.DEV)
            assert t.same_values(hago.mx_dense_grouped(*args, out_dtype=t.OUT[out], out=result), want, t.TYPES[out]), (k, out)


def test_special_cases(kernels):
    for _ in kernels():
        for fmt in ("fp4", "fp8"):
            t.test_dense_of_no_columns_rows_or_features(fmt)
            t.test_dense_blocks_that_are_none(fmt)
            t.test_dense_scales_over_their_range(fmt)
        t.test_grouped_contents_out_of_range_stay_in_bounds()
        t.test_results_do_not_change_from_call_to_call()


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("M,N,K", [(2100, 4200, 256), (1500, 6000, 640), (5000, 1100, 128)])
def test_workgroups_that_go_from_tile_to_tile(kernels, M, N, K, fmt):
    """More tiles than workgroups, ragged at both ends, even and odd numbers of stages; every result against the kernels of few rows."""
    rng = np.random.default_rng(M)
    a, w, bias = t.operand(rng, M, K, fmt, True), t.operand(rng, N, K, "fp4", True), torch.arange(N, dtype=torch.float32, device=t.DEV)
    da, dw = t.on_gpu(a, fmt, K), t.on_gpu(w, "fp4", K)
    want = None
    for k in kernels():
        got = [hago.mx_dense(da, dw, b, out_dtype=o) for b, o in ((bias, hago.F32), (None, hago.BF16))]
        if want is None:
            av, wv = torch.from_numpy(mx.decode(*a, fmt, K)), torch.from_numpy(mx.decode(*w, "fp4", K))
            exact = av.to(t.DEV) @ wv.to(t.DEV).t().contiguous()
            want = [(exact + bias.double()).float(), exact.to(torch.bfloat16)]
        assert all(torch.equal(g, v) for g, v in zip(got, want)), k
