"""The rotary positions and the operators around a paged cache on the CPU, against a runtime that stands in for HIP: statuses, which kernel serves a call, and
launches that hold fewer than 2^32 threads and together enough."""
import re
import subprocess

import pytest

from conftest import build_against_fake_runtime


@pytest.fixture(scope="module")
def lines(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("cache") / "cache_status")
    build_against_fake_runtime("cache_status_driver.cpp", exe)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "cache statuses: ok" in r.stdout, r.stdout[-4000:] + r.stderr
    out = {}
    for line in r.stdout.splitlines():
        if "\t" in line:
            name, launches, kernels = line.split("\t")
            out[name] = ([tuple(map(int, l.split("|"))) for l in launches.split(";") if l], [k for k in kernels.split(";") if k])
    return out


def test_a_refused_launch_is_reported_once(lines):
    assert len(lines) == 19


@pytest.mark.parametrize("name,kernels", [
    ("rope", [r"rope_kernel<1, false>"]), ("write", [r"write_kernel<1, 1, 0, 1>"]), ("write many", [r"write_kernel<1, 1, 0, 2>"]),
    ("read", [r"read_kernel<2, 1, 0, 1>"]), ("read many", [r"read_kernel<2, 1, 0, 2>"]), ("read one column", [r"read_kernel<2, 1, 0, 1>"]),
    ("token", [r"attention_kernel<1, 1, 0, 4, true>", r"join_kernel<1, 4, 4>"]), ("token odd pages", [r"attention_kernel<2, 1, 0, 2, false>", r"join_kernel<2, 2, 4>"]),
    ("prompt", [r"many_kernel<1, 1, 0, 4, 8, true>", r"join_kernel<1, 4, 1>"]), ("prompt odd pages", [r"many_kernel<1, 1, 0, 2, 8, false>", r"join_kernel<1, 2, 1>"]),
    ("prompt wide", [r"many_kernel<2, 1, 0, 8, 4, true>", r"join_kernel<2, 8, 1>"]), ("prompt f32", [r"attention_kernel<0, 1, 0, 4, true>", r"join_kernel<0, 4, 1>"]),
    ("most rows", [r"plan_kernel<16, 128, 2048>", r"attention_kernel<1, 1, 0, 4, true>", r"join_kernel<1, 4, 1>"]), ("many chunks", [r"plan_kernel<256, 64, 256>", r"many_kernel<1", r"join_kernel<1"]),
    ("chunks of sixteen rows", [r"attention_kernel<1, 1, 0, 4, true>", r"join_kernel<1, 4, 4>"])])
def test_which_kernel_serves_a_call(lines, name, kernels):
    got = lines[name][1]
    assert len(got) == len(kernels) and all(re.search(re.escape(k), g) for k, g in zip(kernels, got)), got


def test_launches_hold_fewer_threads_than_one_may(lines):
    for name, (launches, _) in lines.items():
        assert launches and all(0 < grid * block < 2 ** 32 for grid, block in launches), name


@pytest.mark.parametrize("name,T,heads,rows", [("write", 5, 8, 16), ("write many", 100000, 8, 32), ("write most", 2 ** 31 - 1, 65536, 16), ("read", 5, 8, 16),
                                               ("read many", 100000, 8, 32), ("read one column", 100000000, 8, 256), ("read most", 2 ** 31 - 1, 1024, 16)])
def test_every_row_has_a_workgroup(lines, name, T, heads, rows):
    assert sum(grid for grid, _ in lines[name][0]) == -(-T // rows) * heads


@pytest.mark.parametrize("name,rows,tile,seqs,runs,block", [("token", 1 * 4, 16, 1, 2048, 256), ("prompt", 8192 * 4, 256, 1, 256, 512), ("prompt wide", 512 * 4, 128, 1, 256, 256),
                                                            ("most rows", 1 << 27, 16, 1 << 22, 2048, 256)])
def test_every_unit_and_run_has_a_workgroup(lines, name, rows, tile, seqs, runs, block):
    """A tile of rows for every `tile` of them and one more for each sequence, for every head of the cache, and the runs that they may be cut into."""
    heads = 1 if name == "most rows" else 8
    planned = seqs > 256   # (by a launch of one workgroup)
    assert len(lines[name][0]) == 2 + planned and (not planned or lines[name][0][0] == (1, 1024))
    assert lines[name][0][planned] == ((rows // tile + seqs) * heads + runs, block)
