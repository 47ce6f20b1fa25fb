"""Products of so many rows that their workgroups need several launches: every row gets its result."""
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2103_14949_amd as hago

DEV = "cuda:0"
K, N = 128, 16
VALUES = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0.0, -.5, -1, -1.5, -2, -3, -4, -6])


def weights(experts):
    """Feature n of expert e has 4 (n + 1) - e ones and zeros behind them."""
    ones = 4 * torch.arange(1, N + 1)[None] - torch.arange(experts)[:, None]
    codes = torch.zeros(experts, N, K, dtype=torch.uint8)
    codes[torch.arange(K) < ones[..., None]] = 2
    packed = codes[..., 0::2] | codes[..., 1::2] << 4
    return hago.MX(packed.to(DEV), torch.full((experts, N, K // 32), 127, dtype=torch.uint8, device=DEV), hago.MX_FP4, K), ones


def rows_of(T):
    """Row t has the code t % 16 everywhere."""
    codes = (torch.arange(16, dtype=torch.uint8) * 17).to(DEV)[:, None].expand(16, K // 2).repeat(T // 16, 1)
    return hago.MX(codes, torch.full((T, K // 32), 127, dtype=torch.uint8, device=DEV), hago.MX_FP4, K)


def holds(out, ones):
    """out: whole sixteens of rows of one expert."""
    want = (VALUES[:, None] * ones[None]).to(out.dtype).to(DEV)
    for part in out.view(-1, 16, N).split(1 << 20):
        assert bool((part == want).all())


@pytest.fixture
def force():
    torch.cuda.empty_cache()
    yield lambda k: hago.set_test_hook(hago.HOOK_MX_KERNEL, k)
    hago.set_test_hook(hago.HOOK_MX_KERNEL, -1)
    torch.cuda.empty_cache()


# (a workgroup of 1024 threads has 16 rows, one of 256 has 64)
@pytest.mark.timeout(120)
@pytest.mark.parametrize("kernel,T", [(11, (1 << 26) + 48), (3, (1 << 30) + 128)])
def test_dense(force, kernel, T):
    w, ones = weights(1)
    a = rows_of(T)
    out = torch.full((T, N), 77.0, dtype=torch.bfloat16, device=DEV)
    force(kernel)
    hago.mx_dense(a, hago.MX(w.codes[0], w.scales[0], w.fmt, K), out=out)
    holds(out, ones[0])


@pytest.mark.timeout(120)
def test_grouped(force):
    T, ends = (1 << 26) + 48, [0, 16, 1 << 25, (1 << 26) + 48]
    w, ones = weights(3)
    a = rows_of(T)
    out = torch.full((T, N), 77.0, dtype=torch.bfloat16, device=DEV)
    force(11)
    hago.mx_dense_grouped(a, w, torch.tensor(ends, dtype=torch.int32, device=DEV), out=out)
    for e in range(3):
        holds(out[ends[e]:ends[e + 1]], ones[e])
