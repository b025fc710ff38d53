"""Stages that bulk copies fill and threads read by ordinary loads, by reading the sources: such a stage is given back behind a fence between the two
proxies.  The arrival alone orders the reads for other threads' ordinary accesses, not for a bulk copy's writes, which may then overtake them."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_1805_10032_b200", "csrc")


def test_read_stages_are_given_back_behind_a_fence():
    released = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        released += text.count("release_read_stage(")
        for at in re.finditer(r"mbar_arrive\((?:bar_)?c?empty\(", text):        # by hand: a fence within the same few statements
            before = text[max(0, at.start() - 220):at.start()]
            assert "fence.proxy.async" in before and "__syncwarp()" in before, (os.path.basename(path), text[at.start() - 80:at.end() + 20])
            released += 1
    assert released >= 5
    wrapper = re.search(r"void release_read_stage\(.*?\n}", open(os.path.join(CSRC, "zeno_tc.cuh")).read(), re.S).group(0)
    steps = [wrapper.index(s) for s in ("fence.proxy.async", "__syncwarp()", "mbar_arrive(bar)")]
    assert steps == sorted(steps)
