"""What lanes of one wave hand each other through LDS is ordered where it is written and read."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2107_03474_amd", "csrc")


def _function(path, name):
    """The text of a function, comments dropped."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, path)).read())
    at = text.index("{", text.index(" %s(" % name))
    depth, end = 1, at + 1
    while depth:
        depth += {"{": 1, "}": -1}.get(text[end], 0)
        end += 1
    return text[at:end]


def test_a_block_of_values_handed_between_lanes():
    """Append: the stores of a block, what orders them, its loads, and what orders these before the next head's stores."""
    body = _function("layer_paged_append.hip", "turn_values")
    steps = re.findall(r"lds\[[^;]*\] = |wave_lds_sync\(\);|, lds\[", body)
    assert ["store" if "=" in s else "load" if "lds[" in s else "order" for s in steps] == ["store", "order", "load", "order"], steps


def test_the_order_is_a_fence_either_way():
    body = _function("layer_common.h", "wave_lds_sync")
    assert re.findall(r"__ATOMIC_\w+|wave_barrier", body) == ["__ATOMIC_RELEASE", "wave_barrier", "__ATOMIC_ACQUIRE"]
    assert body.count('"wavefront"') == 2
