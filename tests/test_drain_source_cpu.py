"""A CTA that gives up may not hand its shared memory back while copies into it are under way: no run shows that."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2407_18121_b200", "csrc")


def test_the_last_wait_for_copies_does_not_end_with_the_abort_flag():
    """mbar_wait returns as soon as the abort flag is set, which it is by then."""
    found = 0
    for path in glob.glob(os.path.join(CSRC, "*.cu")):
        for block in re.findall(r"if \(\*abort_flag\) \{\n(.*?)\n\s*\}\n", open(path).read(), re.S):
            assert "let copies that are still in flight land" in block
            assert "mbar_drain(" in block and "mbar_wait(" not in block, path
            found += 1
    assert found == 4                                          # importance, prefill attention, chunk attention, chunk weights
    text = open(os.path.join(CSRC, "ec_tc.cuh")).read()
    body = re.search(r"void mbar_drain\(.*?\n\}\n", text, re.S).group(0)
    assert "abort_flag" not in body and "kDrainLimitNs" in body        # bounded all the same
