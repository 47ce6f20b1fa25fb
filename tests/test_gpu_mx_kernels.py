"""Every kernel of the microscaled products, forced in turn, at sizes inside, at and across its tiles."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import paper_2103_14949_amd as hago
import test_gpu_mx as t

KERNELS = range(13)


@pytest.fixture(params=KERNELS)
def kernel(request):
    hago.set_test_hook(hago.HOOK_MX_KERNEL, request.param)
    yield request.param
    hago.set_test_hook(hago.HOOK_MX_KERNEL, -1)


@pytest.mark.parametrize("M,N,K", t.SIZES)
@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_dense(kernel, M, N, K, fmt):
    rng = np.random.default_rng(M + N + K)
    a, w = t.operand(rng, M, K, fmt, True), t.operand(rng, N, K, "fp4", True)
    for out in ("f32", "f16"):
        t.check_dense(a, w, fmt, M, N, K, None, out, exact=True)
    a, w, bias = t.operand(rng, M, K, fmt), t.operand(rng, N, K, "fp4"), rng.standard_normal(N).astype(np.float32)
    t.check_dense(a, w, fmt, M, N, K, bias, "bf16")


@pytest.mark.parametrize("sizes,N,K", t.GROUPS)
@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("gather", [False, True])
def test_grouped(kernel, sizes, N, K, fmt, gather):
    rng = np.random.default_rng(sum(sizes) + N + K)
    bias = rng.standard_normal((len(sizes), N)).astype(np.float32)
    t.check_grouped(t.group_case(rng, sizes, N, K, fmt, gather, True, gap=3), N, K, fmt, None, "f32", True)
    t.check_grouped(t.group_case(rng, sizes, N, K, fmt, gather, False), N, K, fmt, bias, "bf16", False)


def test_special_cases(kernel):
    for fmt in ("fp4", "fp8"):
        t.test_dense_of_no_columns_rows_or_features(fmt)
        t.test_dense_blocks_that_are_none(fmt)
        t.test_dense_scales_over_their_range(fmt)
    t.test_grouped_contents_out_of_range_stay_in_bounds()
    t.test_results_do_not_change_from_call_to_call()
