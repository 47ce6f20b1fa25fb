"""Prepared microscaled calls own the buffers that they write, whatever becomes of the MX that they return."""
import gc
import weakref

import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2103_14949_amd as hago

DEV = "cuda:0"
CALLS = {
    "quantize": lambda x, **k: hago.mx_quantize(x, hago.MX_FP8, prepare=True, **k),
    "rmsnorm": lambda x, **k: hago.mx_rmsnorm(x, prepare=True, **k),
    "silu_mul": lambda x, **k: hago.mx_silu_mul(torch.cat([x, x], 1), hago.MX_FP8, prepare=True, **k),
}


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("values", [False, True])
@pytest.mark.parametrize("name", CALLS)
def test_codes_and_scales_can_be_set_and_the_launch_keeps_its_buffers(name, values, given):
    x = torch.randn(6, 256, generator=torch.Generator().manual_seed(1)).to(DEV)
    room = hago.MX.empty(6, 256, hago.MX_FP8, DEV) if given else None
    call = CALLS[name](x, values=values, out=room)
    mx = call.out[0] if values else call.out
    assert not given or mx is room
    want = CALLS[name](x)()
    alive = weakref.ref(mx.codes), weakref.ref(mx.scales)
    mx.codes, mx.scales = torch.zeros(1, device=DEV), torch.zeros(1, device=DEV)
    gc.collect()
    assert all(r() is not None for r in alive)   # (nothing is launched before this holds)
    call()
    assert torch.equal(alive[0](), want.codes) and torch.equal(alive[1](), want.scales)
    assert float(mx.codes) == 0 and float(mx.scales) == 0
    del call, room
    gc.collect()
    assert all(r() is None for r in alive)       # and not longer than the call is there
