"""Kernels that start beside their predecessor read nothing through the read-only path: what it serves is taken as constant while the
kernel runs, and the compiler may ask for it before the wait for the predecessor."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_14371_b200", "csrc")
SOURCES = sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh")))


def code_of(path):
    with open(path) as f:
        return re.sub(r"//[^\n]*|/\*.*?\*/", "", f.read(), flags=re.S)


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_no_read_only_loads_where_kernels_wait(path):
    code = code_of(path)
    if "pdl_wait();" not in code:
        return
    assert "__ldg(" not in code and "ld.global.nc" not in code
    for kernel in code.split("__global__")[1:]:
        parameters = kernel[: kernel.index("{")]
        if "pdl_wait();" in kernel:
            assert not re.search(r"const\s+\w[\w ]*\*\s*__restrict__", parameters), parameters


def test_the_sources_were_looked_at():
    waiting = {os.path.basename(p) for p in SOURCES if "pdl_wait();" in code_of(p)}
    assert {"lq_norm.cu", "lq_cache_rows.cu", "lq_cache_attend.cuh"} <= waiting
