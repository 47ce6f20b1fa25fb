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
