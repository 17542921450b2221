"""Waits for a barrier's phase go by its parity alone: a thread that waits for the first phase of a barrier that goes on to a second may
come when the second is over, and then waits for ever.  A barrier whose first phase is waited for by name has to have no other."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_14371_b200", "csrc")
SOURCES = [p for p in sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh"))) if "mbarrier.try_wait" in open(p).read()]


def parities(code):
    """Of every barrier of a kernel's shared memory, the parities that it is waited for with, as they are written."""
    code = re.sub(r"//[^\n]*|/\*.*?\*/", "", code, flags=re.S)
    found = {}
    for name, parity in re.findall(r"&sm\.(\w+)(?:\[[^\]]*\])?,\s*((?:[^,()]|\([^()]*\))+)", code):
        if name not in ("failed", "tensor"):
            found.setdefault(name, set()).add(parity.strip())
    return found


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_a_barrier_with_a_first_phase_has_no_second(path):
    for name, given in parities(open(path).read()).items():
        waited = {p for p in given if not re.fullmatch(r"\w*::\w+|32 \* .*|1|readers", p)}      # (barrier_init's counts)
        assert "0" not in waited or waited == {"0"}, (name, waited)


def test_the_waits_were_found():
    assert any(os.path.basename(p) == "lq_cache_shared.cu" for p in SOURCES)
    for path in SOURCES:
        found = parities(open(path).read())
        assert "0" in found["brought"] and any("& 1" in p for p in found["weighed"]) and any("& 1" in p for p in found["key_full"]), found
