"""Inline asm in the kernels.  Between a matrix instruction and a vector instruction that reads what it writes there have to be some cycles.  The compiler sees
to that for its own instructions and not for those in asm, so asm does not compute from the scores."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2510_11062_amd", "csrc")


def test_no_maximum_is_taken_in_asm():
    found = []
    for name in sorted(os.listdir(CSRC)):
        if name.endswith((".hpp", ".hip")):
            text = open(os.path.join(CSRC, name)).read()
            for asm in re.findall(r'\basm\s*(?:volatile\s*)?\(\s*((?:"[^"]*"\s*)+)', text):
                found += [(name, op) for op in re.findall(r"\bv_\w*max\w*", asm)]
    assert not found
