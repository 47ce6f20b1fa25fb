"""The attention's kernel for many rows of bfloat16 queries is written to the registers of two wavefronts a SIMD: the forms of up to 128 columns over pages of whole
eights spill none, as built, and the others a few."""
import glob
import os
import re

import pytest

from paper_2103_14949_amd import build


def test_no_vector_register_is_spilled():
    paths = glob.glob(os.path.join(os.path.dirname(build.LIB), "_build", "mx_attention_many-*gfx950.s"))
    if not paths:
        pytest.skip("no assembly here: the libraries were built elsewhere")
    with open(paths[0]) as f:
        text = f.read()
    kernels = [k for k in re.findall(r"\.name:\s+(\S+).*?\.vgpr_spill_count:\s+(\d+)", text, re.S) if "many_kernel" in k[0]]
    assert len(kernels) == 24 and max(int(spilled) for _, spilled in kernels) <= 16
    assert [k for k, spilled in kernels if int(spilled) and re.search(r"Li[24]ELi8ELb1E", k)] == []


def test_the_file_has_its_flags():
    """Without them the kernel for 256 columns keeps its sums where vector instructions cannot use them."""
    for name in ("mx_attention_many.hip", "mx_attention_many_f16.hip"):
        assert name in build.FILE_FLAGS and os.path.exists(os.path.join(build.CSRC, name))
