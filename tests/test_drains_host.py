"""A block whose wait gave up ends only after the copies and products that it has under way: the
waits before shared memory and TMEM are given back look at no abort flag.  A model of such a block,
and the kernels' source."""
import glob
import os
import random
import re

import pytest

SRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_32525_gb300", "csrc")


def source(name):
    return open(os.path.join(SRC, name)).read()


def leaves_behind(rng, stages, heed_abort, limit=50):
    """A loader with a ring of stages, whose readers have given up: how many of its copies are still
    on their way when it ends.  heed_abort: a drain that gives up at the abort flag, too."""
    issued = rng.randint(1, 4 * stages)
    lands = sorted(rng.randint(0, limit - 1) for _ in range(issued))  # within the drain's own limit
    clock, abort = rng.randint(0, limit // 2), True
    for i in range(max(0, issued - stages), issued):
        if heed_abort and abort and clock < lands[i]:
            clock += 1  # one suspended poll
            continue
        clock = max(clock, lands[i])
    return sum(t > clock for t in lands)


@pytest.mark.parametrize("stages", [2, 3, 4, 6])
def test_a_drain_waits_for_every_copy(stages):
    rng = random.Random(stages)
    assert all(leaves_behind(rng, stages, heed_abort=False) == 0 for _ in range(2000))


def test_one_that_heeds_the_flag_would_not():
    rng = random.Random(0)
    assert sum(leaves_behind(rng, 4, heed_abort=True) > 0 for _ in range(2000)) > 200


def test_the_drain_looks_at_no_flag():
    text = source("fs_tc_ptx.cuh")
    body = re.search(r"void mbar_drain\(uint64_t\* bar, uint32_t parity\) \{\n(.*?)\n\}", text, re.S).group(1)
    assert "Abort" not in body and "flag" not in body and "kWaitNs) return;" in body


def test_kernels_drain_by_it():
    # a wait without a status word was such a drain by the wait that heeds the flag; the one kernel
    # that has no status word waits so for its rows
    for f in glob.glob(os.path.join(SRC, "*.cu*")):
        waits = re.findall(r"mbar_wait(?:_w)?\([^;]*nullptr[^;]*\);", open(f).read())
        assert len(waits) == (2 if f.endswith("fs_rows.cuh") else 0), f
    for f in ("fs_tc_fwd.cu", "fs_tc_bwd.cu", "fs_attn_tc.cuh"):
        text = source(f)
        loaders = len(re.findall(r"for \(int j = \(i > [\w:]+ \? i - [\w:]+ : 0\); j < i; j\+\+\)", text))
        assert loaders and len(re.findall(r"mbar_drain\(&\w*full\[j %", text)) == loaders
        commits = len(re.findall(r"mma_commit_w\(&?drain", text))
        assert commits and len(re.findall(r"mbar_drain_w\(&?drain", text)) == commits
    rows = source("fs_rows.cuh")
    assert len(re.findall(r"mbar_drain\(&full\[i % plan.stages\], \(uint32_t\)\(i / plan.stages\) & 1u\);", rows)) == 1
    assert len(re.findall(r"if \(i < issued\) tc::mbar_drain\(&full\[i\], \(uint32_t\)\(\(issued - 1 - i\) / plan.stages\) & 1u\);", rows)) == 1


@pytest.mark.parametrize("stages", [2, 3, 6])
def test_the_parity_of_a_stages_last_copy(stages):
    """As the two kernels of fs_rows.cuh give it: number i of a block's copies goes to stage i % stages."""
    for issued in range(40):
        copies = [range(s, issued, stages) for s in range(stages)]
        for i in range(max(0, issued - stages), issued):
            assert i == copies[i % stages][-1] and (i // stages) & 1 == (len(copies[i % stages]) - 1) & 1
        for i in range(stages):
            assert (i < issued) == (len(copies[i]) > 0)
            if i < issued:
                assert ((issued - 1 - i) // stages) & 1 == (len(copies[i]) - 1) & 1
