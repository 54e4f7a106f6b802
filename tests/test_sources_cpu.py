"""Rules of the kernels' sources that no run shows when they are broken."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_06763_amd", "csrc")


def test_lds_of_a_wave_is_ordered_by_fences():
    """A wave barrier alone orders nothing in the language's memory model: lanes that exchange values through LDS
    without a workgroup barrier do so behind wave_lds_order(), which has the two fences."""
    found = []
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        text = open(path).read()
        body = re.search(r"void wave_lds_order\(\) \{.*?\n\}", text, re.S)
        if body:
            assert body.group(0).count("__builtin_amdgcn_fence") == 2
            text = text.replace(body.group(0), "")
        found += [os.path.basename(path)] * text.count("__builtin_amdgcn_wave_barrier")
    assert found == []
