"""Serving through the layer around the memory: batches that hold rows of no sequence."""
import pytest
import torch

import paper_2107_03474_amd as lram
from paper_2107_03474_amd.memory_block import KeyValueCache, MemoryBlock

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_padded_batches():
    torch.manual_seed(3)
    block = MemoryBlock(128, 4, (4,) * 8, 2, True, buckets=16, reach=20, table_dtype=torch.float32).eval()
    with torch.no_grad():
        block.bias.normal_()
    plain, padded = (KeyValueCache(2, 32, 2, 32, torch.float32) for _ in range(2))
    for step in ([12, 3], [1, 1], [0, 5], [7, 9]):
        x = torch.randn((sum(step), 128), device=DEV)
        want = block.serve(x, lram.pack(step), plain)
        more = torch.cat([torch.full((2, 128), 9.0, device=DEV), x, torch.full((5, 128), 7.0, device=DEV)])
        seqs = lram.pack(step)
        got = block.serve(more, seqs._replace(start_q=seqs.start_q + 2), padded)
        # the same rows among others: the projections may sum in another order
        assert (got[2:-5] - want).abs().max() < 2e-4
        assert torch.equal(plain.used, padded.used)
    with pytest.raises(ValueError, match="capacity"):
        block.serve(torch.randn((14, 128), device=DEV), lram.pack([13, 1]), plain)
    assert plain.used.tolist() == [20, 18]
