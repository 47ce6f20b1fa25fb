"""Launches of the microscaled products, on the CPU: none has 2^32 threads, and together they cover every tile once."""
import re
import subprocess

import pytest

from conftest import build_against_fake_runtime


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("mx_launches") / "mx_launches")
    build_against_fake_runtime("mx_launch_driver.cpp", exe)

    def run(lines):
        r = subprocess.run([exe], input="".join(line + "\n" for line in lines), capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stderr
        out = []
        for line in r.stdout.splitlines():
            status, *launches, name = line.split("\t")
            out.append((int(status), [tuple(map(int, l.split("|"))) for l in launches], name))
        return out
    return run


def shape(name):
    """Features, rows and threads of a kernel's tile, and whether its workgroups go from tile to tile."""
    kind, args = re.search(r"mx_(few|tile)_kernel<([^>]*)>", name).groups()
    n = [int(v) for v in args.split(",") if v.strip() not in ("true", "false")]
    if kind == "few":
        return 16 * n[1], 16 * n[2], None, False
    _, wp, wq, tp, tq, slots, _ = n
    return wp * tp * 32, wq * tq * 32, 64 * wp * wq, tp % 2 == 0 and slots == 2 and tp * tq < 8


def check(line, answer):
    status, launches, name = answer
    kind, _, _, rows, *rest = line.split()
    experts, features = (int(rest[0]), int(rest[1])) if kind == "grouped" else (None, int(rest[0]))
    rows = int(rows)
    assert status == 0 and launches, line
    bp, bq, threads, stays = shape(name)
    row_tiles = -(-rows // bq) if experts is None else min(rows, rows // bq + experts)
    tiles = -(-features // bp) * row_tiles
    for grid, block, _ in launches:
        assert 0 < grid * block < 2 ** 32 and (threads is None or block == threads), line
    if stays:
        assert [(g, a) for g, _, a in launches] == [(launches[0][0], launches[0][0])] and launches[0][0] <= tiles, line
        return
    at = 0
    for grid, _, first in launches:
        assert first == at and first % 8 == 0, line   # (an eighth of the tiles belongs to an XCD)
        at += grid
    assert at == tiles, line


LARGE = ["dense -1 0 1073741824 16 128", "dense -1 0 268435456 16 512", "dense -1 1 1 1073741824 128", "grouped -1 1 262144 262144 4096 128",
         "grouped -1 0 1073741824 4 16 128", "dense -1 1 2147483391 16 128", "dense -1 0 16 2147483391 128"]


def test_launches_of_the_largest_products(ask):
    for line, answer in zip(LARGE, ask(LARGE)):
        check(line, answer)


def test_launches_of_every_kernel(ask):
    lines = [f"dense {k} {f} {m} {n} 256" for k in range(13) for f in (0, 1) for m, n in
             ((1, 1), (17, 33), (300, 515), (8192, 8192), (1 << 26, 16), ((1 << 26) + 1, 33), (16, 1 << 28), (1 << 30, 16), (5, (1 << 30) + 7))]
    lines += [f"grouped {k} {f} {t} {e} {n} 128" for k in range(13) for f in (0, 1) for t, e, n in ((1, 1, 16), (64, 3, 100), (16384, 32, 4096), (1 << 22, 1 << 22, 256))]
    for line, answer in zip(lines, ask(lines)):
        check(line, answer)
