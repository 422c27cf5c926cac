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
