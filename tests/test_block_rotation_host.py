"""What a rotating MemoryBlock refuses when it is built.  No GPU is needed."""
import math

import pytest
import torch

import paper_2107_03474_amd as lram
from paper_2107_03474_amd.memory_block import MemoryBlock


def _block(w, heads, kv_heads, rotary):
    return MemoryBlock(w, heads, (2,) * 8, kv_heads, device="cpu", rotary=rotary)


def test_what_no_call_could_run():
    plan = lram.rotary_plan(32, device="cpu")
    with pytest.raises(ValueError, match="at most 64 times"):
        _block(65 * 32, 65, 1, plan)
    assert _block(64 * 32, 64, 1, plan).kv_heads == 1
    for magnitude in (math.inf, math.nan):
        with pytest.raises(ValueError, match="magnitude must be finite"):
            _block(128, 4, 4, plan._replace(magnitude=magnitude))
    for turns in (plan.turns.double(), plan.turns.to(torch.int32), plan.turns[None]):
        with pytest.raises(ValueError, match="int64"):
            _block(128, 4, 4, plan._replace(turns=turns))
    for turns in (plan.turns[:0], torch.zeros(17, dtype=torch.int64)):
        with pytest.raises(ValueError, match="1 to head_dim / 2 pairs"):
            _block(128, 4, 4, plan._replace(turns=turns))
