"""That the batches of attention_cases.py are served by the kernel for many rows, and planned in front where they have many sequences; on the CPU."""
import subprocess

import pytest

import paper_2103_14949_amd as hago
from attention_cases import CUT, PLANNED, tokens
from conftest import build_against_fake_runtime

TYPES = {"f32": 0, "bf16": 1, "f16": 2}


@pytest.fixture(scope="module")
def serve(tmp_path_factory):
    """Calls (type, T, heads, kv_heads, dim, seqs, page) -> their kernels, and the bytes of their workspaces."""
    exe = str(tmp_path_factory.mktemp("attention") / "routes")
    build_against_fake_runtime("attention_route_driver.cpp", exe)

    def kernels(calls):
        r = subprocess.run([exe], input="".join(" ".join(map(str, c)) + "\n" for c in calls), capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stderr
        lines = [line.split("\t") for line in r.stdout.splitlines()]
        assert len(lines) == len(calls)
        return [([k for k in names.split(";") if k], int(n)) for names, n in lines]
    return kernels


@pytest.mark.parametrize("case", CUT + PLANNED)
def test_the_kernel_for_many_rows_serves_them(serve, case):
    (kernels, _), = serve([(TYPES[case.get("name", "bf16")], tokens(case), case["heads"], case["kv_heads"], case["dim"], len(case["new"]), case["page"])])
    planned = len(case["new"]) > 256
    assert len(kernels) == 2 + planned and "many_kernel<" in kernels[planned] and "join_kernel<" in kernels[-1]
    assert not planned or "plan_kernel<" in kernels[0]


@pytest.mark.parametrize("case", CUT + PLANNED)
def test_some_of_their_sequences_are_cut(case):
    """Units (a tile of rows, a head) and their blocks of 64 keys: about 256 runs share all blocks, and a unit of more than a share is cut."""
    rows = 32 * (8 if case.get("name", "bf16") == "bf16" and case["dim"] <= 128 else 4)
    units, blocks = [], []
    for n, length in zip(case["new"], case["lengths"]):
        low = max(0, length - n - case["window"] + 1) if case.get("window") else 0
        units.append(-(-n * (case["heads"] // case["kv_heads"]) // rows) * case["kv_heads"])
        blocks.append(-(-(length - low // 16 * 16) // 64))
    share = -(-sum(u * b for u, b in zip(units, blocks)) // 256)
    runs = [-(-b // share) for u, b in zip(units, blocks) if u]
    assert max(runs) > 1
    assert len(case["new"]) == 1 or case in CUT or min(runs) == 1


@pytest.mark.parametrize("heads,kv_heads,dim", [(32, 8, 128), (4, 4, 64), (16, 1, 256)])
def test_room_for_the_largest_call_serves_the_smaller_ones(serve, heads, kv_heads, dim):
    """Whichever kernel each of them has: the size does not fall where tokens or sequences rise, and a call takes as much as the size says."""
    sizes = [(T, seqs) for T in (1, 8, 9, 32, 33, 64, 300, 5000) for seqs in (1, 2, 64, 256, 257, 300)]
    bytes_of = {s: hago.mx_attention_workspace_bytes(*s, heads, kv_heads, dim) for s in sizes}
    for a in sizes:
        assert all(bytes_of[b] >= bytes_of[a] for b in sizes if b[0] >= a[0] and b[1] >= a[1])
    got = serve([(t, T, heads, kv_heads, dim, seqs, 64) for t in (0, 1, 2) for T, seqs in sizes])
    assert [n for _, n in got] == 3 * [bytes_of[s] for s in sizes]
    assert {"many_kernel" in k[-2] for k, _ in got} == {True, False}
