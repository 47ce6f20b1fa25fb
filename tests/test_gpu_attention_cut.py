"""The kernel for many rows where sequences are cut into runs and joined, planned in front or not, on the GPU against the oracle."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2103_14949_amd as hago
from attention_cases import CUT, PLANNED, ROWS_BEFORE, ROWS_BEHIND
from cache_util import DEV, layout, on_gpu, random_cache
from test_gpu_mx_attention import run


@pytest.mark.parametrize("case", CUT + PLANNED)
def test_cut_sequences(case):
    run(**case, seed=17, rows_before=ROWS_BEFORE, rows_behind=ROWS_BEHIND)


@pytest.mark.parametrize("case", PLANNED)
def test_the_same_twice_and_in_a_graph(case):
    """Bit by bit the same, eager and replayed, with workspaces of other contents between."""
    rng = np.random.default_rng(3)
    table, lengths, offsets, pages = layout(case["new"], case["lengths"], case["page"])
    dtype = {"bf16": torch.bfloat16, "f16": torch.float16}[case.get("name", "bf16")]
    cache, _, _ = random_cache(rng, pages, case["kv_heads"], case["page"], case["dim"], case.get("k_fmt", "fp8"), case.get("v_fmt", "fp8"))
    where = on_gpu(table, lengths, offsets)
    T = int(offsets[-1])
    q = torch.randn(T, case["heads"], case["dim"], device=DEV, dtype=dtype)
    call = dict(causal=case.get("causal", True), window=case.get("window", 0), lse=True)
    want = hago.mx_attention(q, cache, *where, **call)
    room = torch.empty(hago.mx_attention_workspace_bytes(T, len(lengths), case["heads"], case["kv_heads"], case["dim"]), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replayed = hago.mx_attention(q, cache, *where, workspace=room, **call)
    for byte in (0, 0x7F, 0xFF):
        room.fill_(byte)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, want))
        assert all(torch.equal(a, b) for a, b in zip(hago.mx_attention(q, cache, *where, **call), want))


def test_offsets_that_break_the_contract():
    """Nothing out of range is touched, and every call ends: planned, and by the kernel for many rows."""
    cache = hago.MXCache.empty(8, 1, 16, 32)
    for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales):
        t.zero_()
    q = torch.randn(700, 16, 32, device=DEV, dtype=torch.bfloat16)
    for bad in ([0, 700, 5], [-3, 2 ** 31 - 1], [700, 350, 0], [2 ** 31 - 1, -2 ** 31]):
        off = np.resize(np.array(bad, np.int32), 301)
        for length in (30, 2 ** 31 - 1, -5):
            hago.mx_attention(q, cache, *on_gpu(np.zeros((300, 2), np.int32), np.full(300, length, np.int32), off))
    torch.cuda.synchronize()
