"""The ring of records that linear_tc.cu's warps go by, as the source has it: a record is
written again once every warp that reads it has said so.  No result shows a reader
that is not waited for, only its place in the time of a call.  No GPU needed."""
import os
import re

import paper_2607_25852_gb300 as spec

CSRC = os.path.join(os.path.dirname(spec.__file__), "csrc")


def kernel():
    with open(os.path.join(CSRC, "linear_tc.cu")) as f:
        source = re.sub(r"//[^\n]*", lambda m: m.group() if "----" in m.group() else "", f.read())
    begin = source.index("linear_tc_kernel(")
    return source[begin:source.index("linear_scan_kernel")]


ROLES = {  # its begin in the source: warps where outputs are made, where only states are
    "---- P: row": (4, 0), "---- loads,": (2, 2), "---- MMAs": (1, 1), "---- the list:": (1, 1), "---- V': half": (8, 8),
    "---- the state:": (8, 8), "---- O: value": (8, 0)}


def roles():
    source = kernel()
    at = sorted((source.index(name), name) for name in ROLES)
    ends = [a for a, _ in at[1:]] + [len(source)]
    return {name: source[a:end] for (a, name), end in zip(at, ends)}


def test_every_reader_of_a_record_is_waited_for():
    # warps: 32 where outputs are made; 24 otherwise, of which 4 have no part
    assert [sum(w[k] for w in ROLES.values()) for k in (0, 1)] == [32, 20]
    count = re.search(r"mbar_init\(&ctl\.used\[s\], (\d+) \+ kWeighers \+ (\d+) \+ \(kOut \? (\d+) \+ (\d+) : 0\)\);",
                      kernel())
    weighers = 8
    always, more = int(count[1]) + weighers + int(count[2]), int(count[3]) + int(count[4])
    readers = [sum(w[k] for name, w in ROLES.items() if "list" not in name) for k in (0, 1)]
    assert [always + more, always] == readers


def test_every_reader_arrives_for_every_record():
    for name, source in roles().items():
        if "list" in name:
            continue
        loop = source[re.search(r"while \(const Record\* r = next\(\)\) \{|for \(; ok; \+\+c\) \{", source).end():]
        if "MMAs" in name:  # one thread, which needs no more than two fields, at the loop's begin
            arrive = loop.index("mbar_arrive(&ctl.used[c % kRecords]);")
            assert "if (" not in loop[:arrive].replace("if (!ok) break;", "")
            assert "ctl.records" not in loop[arrive:]
            continue
        assert loop.count("done();") == 1 and "ctl.used" not in loop
        # nothing but a wait that gave up leaves the loop, or begins it anew, before
        before = loop[:loop.index("done();")]
        assert "continue" not in re.sub(r"if \(!kOut \|\| \(pass && ends\)\) continue;|if \(!bf16_not_finite\(\*value\)\) continue;",
                                        "", before)
        assert not re.search(r"(?<!if \(!ok\) )break;", before)


def in_flight(ahead, stages):
    """A loading warp's chunks that may still be on their way where it gives up at its next one, every stage filled as
    early as the ring lets it: chunk x once x - stages was read, and those are read in order."""
    return [x for x in range(ahead - 2, -1, -2) if x + stages >= ahead]


def test_copies_in_flight_end_before_the_cta():
    """Where a wait gives up the boxes that the loading warps have sent are waited for, with a limit, before the CTA
    ends; the MMAs' products by their thread."""
    source = roles()
    loop = source["---- loads,"]
    loop = loop[loop.index("while (const Record* r = next())"):]
    # noted after the last wait that may give up, before the first box
    assert loop.index("if (!ok) break;") < loop.index("ctl.sent[warp & 1] = chunk + 1;") < loop.index("bring(&tmQ")
    end = source["---- O: value"]
    end = end[end.index("__syncthreads();"):]
    drain = re.search(r"for \(uint32_t x = 0; x < 4; \+\+x\) \{\s*const uint32_t sent = ctl\.sent\[x & 1\], y = 1 \+ \(x & 2\);\s*"
                      r"if \(y <= sent\) wait_phase\(&ctl\.full\[\(sent - y\) % kStages\], \(sent - y\) / kStages & 1u, p\.status\);", end)
    assert drain and "if (tid == 0 && ctl.aborted) {" in end[:drain.start()]
    for stages in (3, 4):
        for ahead in range(2, 40):  # `sent` is ahead - 1
            waited = [ahead - 1 - y for y in (1, 3) if y <= ahead - 1]
            assert set(in_flight(ahead, stages)) <= set(waited)
            # none of their barriers is two uses on, where the wait would be for another chunk: the other warp's chunks
            # end below ahead + stages, as nothing from `ahead` on is read, and this warp's below `ahead`
            assert all(x + 2 * stages >= ahead + stages or (x + 2 * stages - ahead) % 2 == 0 for x in waited)
    assert "wait_phase(&ctl.drained, 0u, p.status);" in source["---- MMAs"]
