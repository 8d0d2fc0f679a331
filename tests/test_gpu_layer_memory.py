"""What the layer's operators allocate."""
import pytest
import torch

import paper_2107_03474_amd as lram

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _allocations(f):
    f()
    torch.cuda.synchronize()
    before = torch.cuda.memory_stats()["allocation.all.allocated"]
    keep = f()
    return torch.cuda.memory_stats()["allocation.all.allocated"] - before, keep


def test_norm_keeps_nothing_for_a_backward_that_cannot_come():
    x, r = (torch.randn((30, 64), device=DEV) for _ in range(2))
    w, b = torch.ones(64, device=DEV, requires_grad=True), torch.zeros(64, device=DEV)
    with torch.no_grad():
        n, y = _allocations(lambda: lram.layer_norm(x, w, b))
        assert n == 1
        n, (y2, h) = _allocations(lambda: lram.layer_norm(x, w, b, residual=r))
        assert n == 2
    full = lram.layer_norm_forward(x, w.detach(), b, residual=r)
    assert torch.equal(y2, full[0]) and torch.equal(h, full[1])
    assert torch.equal(y, lram.layer_norm_forward(x, w.detach(), b)[0])
    n, _ = _allocations(lambda: lram.layer_norm(x, w, b))
    assert n == 3  # with a backward to come: the statistics too
