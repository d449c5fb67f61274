"""What the warps of the tree attention wait for, as far as it can be told without a GPU."""
import glob
import os
import re

from conftest import ROOT

CSRC = os.path.join(ROOT, "paper_2607_21042_b200", "csrc")


def test_a_look_at_a_barrier_has_one_answer_for_the_warp():
    """Lanes that poll a barrier while others arrive may see different things.  Where votes of all lanes follow, a branch on a lane's own answer could leave some of them
    behind for good, so that what looks without waiting votes itself."""
    found = 0
    for path in glob.glob(os.path.join(CSRC, "*.cuh")):
        text = open(path).read()
        for at in (m.start() for m in re.finditer(r"mbarrier\.test_wait", text)):
            found += 1
            body = text[at:text.index("\n}", at)]
            assert re.search(r"return __(any|all)_sync\(0xFFFFFFFFu, done != 0\);", body), (path, body)
    assert found


def test_the_end_of_a_range_is_the_warps():
    """The error word decides whether a CTA has work; other warps may set it meanwhile, and the loop over the range votes."""
    text = open(os.path.join(CSRC, "attention_tree.cuh")).read()
    decisions = re.findall(r"u_end = ([^;]*\?)", text)
    assert decisions == ["__any_sync(0xFFFFFFFFu, *failed) ?"]
