"""The attention's kernels for many rows as they were built, of bfloat16 and float16 queries."""
import glob
import os
import re

import pytest

from paper_2103_14949_amd import build

FILES = ["mx_attention_many", "mx_attention_many_f16"]


def assembly(name):
    paths = glob.glob(os.path.join(os.path.dirname(build.LIB), "_build", name + "-*gfx950.s"))
    if not paths:
        pytest.skip("no assembly here: the libraries were built elsewhere")
    with open(paths[0]) as f:
        return f.read()


@pytest.mark.parametrize("name", FILES)
def test_rows_in_lds_are_written_whole(name):
    """Sixteen bytes at an address of sixteen: where the compiler sees another, it writes two halves."""
    text = assembly(name)
    assert "ds_write_b128" in text and "ds_write2_b64" not in text and "ds_write2st64_b64" not in text


@pytest.mark.parametrize("name,most", [("mx_attention_many", 16), ("mx_attention_many_f16", 84)])
def test_registers(name, most):
    """No form over pages of whole eights (sixteens) and up to 128 columns spills a vector register, and of float16 queries none of any columns; others as many as the design notes
    say."""
    kernels = re.findall(r"\.name:\s+(\S*many_kernelI\S+).*?\.vgpr_spill_count:\s+(\d+)", assembly(name), re.S)
    assert len(kernels) == 24 and max(int(n) for _, n in kernels) <= most
    whole = "Li[24]ELi[48]ELb1E" if name == "mx_attention_many" else "ELb1E"
    assert [k for k, n in kernels if int(n) and re.search(whole, k)] == []
