"""Offsets that break the contract so that they stand for 2^31 tiles and more: the call ends, and nothing beside its results is written."""
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2103_14949_amd as hago

DEV = "cuda:0"
K, N = 128, 16


@pytest.mark.timeout(120)
@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("kernel,log_rows,log_experts", [(11, 25, 13), (10, 25, 14), (4, 25, 13), (3, 25, 14), (2, 25, 14), (1, 26, 14), (0, 26, 14)])
def test_groups_that_are_all_rows(kernel, log_rows, log_experts, fmt):
    T, E = 1 << log_rows, 1 << log_experts
    code = hago.MX_FP4 if fmt == "fp4" else hago.MX_FP8
    full = lambda value, *shape: torch.full(shape, value, dtype=torch.uint8, device=DEV)  # noqa: E731
    a = hago.MX(full(0x22 if fmt == "fp4" else 0x38, T, K // 2 if fmt == "fp4" else K), full(127, T, K // 32), code, K)   # ones
    w = hago.MX(full(0x22, E, N, K // 2), full(127, E, N, K // 32), hago.MX_FP4, K)
    offsets = torch.zeros(E + 1, dtype=torch.int32, device=DEV)
    offsets[1::2] = T
    keep = torch.full((T + 64, N), 77.0, dtype=torch.bfloat16, device=DEV)
    hago.set_test_hook(hago.HOOK_MX_KERNEL, kernel)
    try:
        hago.mx_dense_grouped(a, w, offsets, out=keep[:T])
        torch.cuda.synchronize()
    finally:
        hago.set_test_hook(hago.HOOK_MX_KERNEL, -1)
    assert bool((keep[T:] == 77).all())
    assert bool((keep[:T] == 128).all())   # (every group has the same weights, and the first one all rows)
    torch.cuda.empty_cache()
