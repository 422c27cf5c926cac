"""The waits of spec_attend's softmax warps, as the source has them.

What follows such a wait (tcgen05.ld, the named barriers) has to be executed by
a warp as one, and a loop that each lane leaves by itself does not promise
that; no result shows it.  So the waits end by a vote of the warp.  No GPU
needed."""
import os
import re

import pytest

import paper_2607_25852_gb300 as spec

CSRC = os.path.join(os.path.dirname(spec.__file__), "csrc")


@pytest.mark.parametrize("name", ["attend_tc.cu", "attend_rows.cu"])
def test_softmax_waits_end_by_a_vote(name):
    with open(os.path.join(CSRC, name)) as f:
        source = f.read()
    begin, end = source.index("// ---- softmax ----"), source.index("// ---- MMAs ----")
    waits = re.findall(r"[^\n]*wait_phase\(", source[begin:end])
    assert waits
    assert all(re.search(r"__all_sync\(0xFFFFFFFFu, wait_phase\($", w) for w in waits), waits


def test_warps_converge_before_tensor_memory_instructions():
    """Likewise past code that lanes leave apart: the item's end, and values that rows must not see."""
    def source(name):
        with open(os.path.join(CSRC, name)) as f:
            return re.sub(r"//[^\n]*", "", f.read())
    rows, few = source("attend_rows.cu"), source("attend_tc.cu")
    assert re.search(r"__syncwarp\(\);\s*tmem_ld32\(my_o \+ d, o\);\s*if \(!real\) continue;", rows)
    assert re.search(r"hide_values<D>\([^;]*;\s*proxy_fence\(\);\s*__syncwarp\(\);", rows)
    assert re.search(r"for_edge_values\(.*?\}\);\s*__syncwarp\(\);", few, re.S)
