"""What the kernels' sources promise the compiler."""
import glob
import os
import re

import paper_2405_18400_amd as pkg


def test_inline_assembly_names_the_registers_that_it_writes():
    """An asm statement that sets M0 names it as lost."""
    found = 0
    for path in glob.glob(os.path.join(os.path.dirname(pkg.__file__), "csrc", "*.h*")):
        text = open(path).read()
        for statement in re.findall(r"\basm(?:\s+volatile)?\s*\(.*?\);", text, re.S):
            if re.search(r"\bs_mov_b32 m0\b", statement):
                found += 1
                assert re.search(r':[^:]*"m0"\s*\)\s*;$', statement), (path, statement)
    assert found
