"""A block's rotation in its state: saved and loaded whole, and its own.  No GPU is needed."""
import copy

import pytest
import torch

import paper_2107_03474_amd as lram
from paper_2107_03474_amd.memory_block import MemoryBlock


def _plan(dim=32, **kw):
    return lram.rotary_plan(dim, device="cpu", **kw)


def _block(rotary):
    return MemoryBlock(128, 2, (2,) * 8, device="cpu", rotary=rotary)


def _of(block):
    plan, bias = block._positions()
    assert bias is None
    return plan.turns.tolist(), plan.interleaved, plan.magnitude


SCALED = dict(interleaved=True, scaling="parts", factor=8.0, length=2048)


@pytest.mark.parametrize("how", [dict(), dict(assign=True), dict(strict=False)], ids=str)
def test_a_saved_rotation_is_loaded_whole(how):
    scaled, plain = _plan(**SCALED), _plan()
    saved, block = _block(scaled), _block(plain)
    state = copy.deepcopy(saved.state_dict())
    assert all(isinstance(t, torch.Tensor) for t in state.values())
    got = block.load_state_dict(state, **how)
    assert not got.missing_keys and not got.unexpected_keys
    assert _of(block) == _of(saved) == (scaled.turns.tolist(), True, scaled.magnitude)
    back = _block(scaled)
    back.load_state_dict(_block(plain).state_dict(), **how)
    assert _of(back) == (plain.turns.tolist(), False, 1.0)


def test_inside_another_module():
    layers, others = (torch.nn.ModuleList([_block(p) for p in plans]) for plans in ((_plan(**SCALED), _plan()), (_plan(), _plan(base=100.0))))
    others.load_state_dict(layers.state_dict())
    assert [_of(b) for b in others] == [_of(b) for b in layers]


def test_frequencies_without_the_rest_of_another_rotation():
    """A state that holds turns alone: taken where they are the block's own, to a double's rounding, and reported otherwise."""
    plan = _plan(**SCALED)
    block = _block(plan)
    state = block.state_dict()
    del state["rotation"]
    state["turns"] = state["turns"] + torch.arange(-8, 8) * 300
    block.load_state_dict(state)
    assert _of(block) == (state["turns"].tolist(), True, plan.magnitude)
    with pytest.raises(RuntimeError, match='Missing key.*"rotation"'):
        _block(_plan()).load_state_dict(state)
    half = _block(_plan(base=50.0, **SCALED))
    state["turns"] = half.turns ^ -(1 << 63)  # half a turn away: the difference has no size of its own
    with pytest.raises(RuntimeError, match='Missing key.*"rotation"'):
        half.load_state_dict(state)


def test_frequencies_are_the_blocks_own():
    plan = _plan()
    first, second = _block(plan), _block(plan)
    before = plan.turns.tolist()
    first.load_state_dict(_block(_plan(base=77.0)).state_dict())
    first.turns.add_(5)
    assert plan.turns.tolist() == before == second.turns.tolist()


def test_a_state_without_a_rotation():
    """A block with a bias keeps its names, and the two kinds do not load each other."""
    bias = MemoryBlock(128, 2, (2,) * 8, device="cpu")
    assert not {"turns", "rotation"} & set(bias.state_dict())
    bias.load_state_dict(MemoryBlock(128, 2, (2,) * 8, device="cpu").state_dict())
    block = _block(_plan(**SCALED))
    with pytest.raises(RuntimeError, match='(?s)Missing key.*"bias".*Unexpected key.*"rotation"'):
        bias.load_state_dict(block.state_dict())
    with pytest.raises(RuntimeError, match='(?s)Missing key.*"rotation"'):
        block.load_state_dict(bias.state_dict())
    other = _block(_plan(16))
    with pytest.raises(RuntimeError, match="size mismatch"):
        other.load_state_dict(block.state_dict())
    assert _of(other) == _of(_block(_plan(16)))
    state = block.state_dict()
    state["rotation"] = torch.zeros(3)
    with pytest.raises(RuntimeError, match="rotation"):
        block.load_state_dict(state)
