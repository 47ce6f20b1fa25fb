"""Microscaled entry points on the CPU, against a runtime that stands in for HIP."""
import subprocess

import pytest

from conftest import build_against_fake_runtime


@pytest.fixture(scope="module")
def lines(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("mx") / "mx_status")
    build_against_fake_runtime("mx_status_driver.cpp", exe)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "microscaled statuses: ok" in r.stdout, r.stdout[-4000:] + r.stderr
    return dict(line.split("\t") for line in r.stdout.splitlines() if "\t" in line)


def test_a_refused_launch_is_reported_once(lines):
    assert len(lines) == 7


@pytest.mark.parametrize("name,kernel", [
    ("quantize", "mx_quantize_kernel<1, 0, false>"), ("silu_mul", "mx_quantize_kernel<0, 1, true>"),
    ("rmsnorm", "mx_rmsnorm_kernel<2, 1, 1, 0>"), ("rmsnorm short", "mx_rmsnorm_kernel<0, 1, 1, 16>"),
    ("dense few", "mx_few_kernel<1"), ("dense large", "mx_tile_kernel<0, 2, 4, 4, 2"), ("grouped", "mx_tile_kernel<1, 2, 4, 4, 2, 3")])
def test_which_kernel_serves_a_call(lines, name, kernel):
    assert kernel in lines[name], lines[name]
