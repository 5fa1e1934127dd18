"""Dependent launches, read from the sources: the decode attention loads lengths, tables and cache tiles before its own
wait, on the ground that the launch before it lets it start only behind that launch's own wait (or on completion)."""
from __future__ import annotations

import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_27269_gb300", "csrc")

# The decode attention itself lets its dependents (the combine, the next projection) start at once; a page plan's only
# dependent is the launch that copies for it, which waits.
AT_ONCE = {"attn_tc.cu": 1, "gqa.cu": 1, "pages.cu": 2}


@pytest.mark.parametrize("name", sorted(os.path.basename(f) for f in glob.glob(os.path.join(CSRC, "*.cu"))))
def test_dependents_start_behind_the_kernels_own_wait(name):
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    early = 0
    for kernel in text.split("__global__")[1:]:
        waited = False
        for call in re.findall(r"griddep_(wait|launch_dependents)\(\)", kernel):
            waited = waited or call == "wait"
            early += call == "launch_dependents" and not waited
    assert early == AT_ONCE.get(name, 0)
