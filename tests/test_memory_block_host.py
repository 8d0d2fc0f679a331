"""What MemoryBlock refuses when it is built."""
import pytest
import torch

from paper_2107_03474_amd.memory_block import MemoryBlock


def _block(w, heads, kv_heads=None, **kw):
    return MemoryBlock(w, heads, (2,) * 8, kv_heads, device="cpu", **kw)


@pytest.mark.parametrize("w,heads", [(96, 2), (64, 4), (512, 2), (160, 2)])
def test_head_width(w, heads):
    with pytest.raises(ValueError, match="32, 64 or 128"):
        _block(w, heads)


def test_bias():
    for w, heads, kv, kw in ((16 * 32, 16, 1, {}), (64 * 32, 64, 1, dict(reach=1)), (128, 4, 2, dict(buckets=257)),
                             (128, 4, 4, dict(reach=1952)), (128, 1, 1, dict(reach=587))):
        with pytest.raises(ValueError, match="2 reach|256 buckets"):
            _block(w, heads, kv, **kw)
    assert _block(9 * 32, 9, 1).bucket.numel() == 257
    assert _block(16 * 32, 16, 1, reach=31).bucket.numel() == 63
    assert _block(128, 1, 1, reach=587, dtype=torch.bfloat16).bucket.numel() == 1175


def test_heads():
    with pytest.raises(ValueError, match="multiple"):
        _block(100, 3)
    with pytest.raises(ValueError, match="multiple"):
        _block(128, 4, 3)
