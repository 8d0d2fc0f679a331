"""What the compiler is told about inline assembly."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2107_03474_amd", "csrc")


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.hip"))),
                         ids=os.path.basename)
def test_m0_is_named_where_it_is_written(path):
    """A statement that writes m0 says so, so that no value of the compiler's is kept there across it."""
    for asm in re.findall(r"asm volatile\((.*?)\);", open(path).read(), flags=re.S):
        text, _, rest = asm.partition(":")
        if re.search(r"\bm0\b", text):
            assert '"m0"' in rest.split(":")[-1], asm


def test_the_statements_are_found():
    text = open(os.path.join(CSRC, "layer_attention.h")).read()
    assert len([a for a in re.findall(r"asm volatile\((.*?)\);", text, flags=re.S) if "s_mov_b32 m0" in a]) == 2
