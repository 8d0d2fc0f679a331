"""The cache's calls inside a level of forward-mode derivatives: only a tangent is refused."""
import pytest
import torch
from torch.autograd import forward_ad

import paper_2107_03474_amd as lram


def _calls(device):
    keys, table = lram.paged_keys(4, 2, 32, 32, torch.float32, device=device), lram.page_table(1, 2, device=device)
    table.table.copy_(torch.tensor([[2, 0]]))
    seqs = lram.pack([3], device=device)._replace(max_k=3)
    rows = torch.randn((3, 2, 32), device=device)
    bias = lram.RelativeBias(torch.zeros((2, 2), device=device), torch.tensor([0, 0, 1], dtype=torch.int32, device=device))

    def append(k=rows, v=rows, q=rows):
        return lram.paged_append(k, v, keys, table, seqs, q=q)

    def attend(q=rows, weight=bias.weight):
        return lram.paged_attention(q, keys, table, seqs, rel=bias._replace(weight=weight))

    return append, attend, rows, bias.weight, table, seqs


def test_what_is_refused():
    append, attend, rows, weight, _, _ = _calls("cpu")
    for call in (append, attend):
        with forward_ad.dual_level(), pytest.raises(lram.LramError, match="GPU tensor"):  # by what comes after
            call()
    with forward_ad.dual_level():
        x, w = (forward_ad.make_dual(t, torch.ones_like(t)) for t in (rows, weight))
        for call in (lambda: append(k=x), lambda: append(v=x), lambda: append(q=x), lambda: attend(q=x), lambda: attend(weight=w)):
            with pytest.raises(lram.LramError, match="no gradients"):
                call()
            with torch.no_grad(), pytest.raises(lram.LramError, match="no gradients"):  # which keeps tangents
                call()


@pytest.mark.gpu
def test_without_a_tangent():
    append, attend, rows, _, table, seqs = _calls("cuda")
    lram.paged_extend(table, seqs)
    append()
    want = attend()
    with forward_ad.dual_level():
        assert append() is rows
        assert torch.equal(attend(), want)
        with torch.no_grad():
            assert torch.equal(attend(rows.clone().requires_grad_()), want)
        with pytest.raises(lram.LramError, match="no gradients"):
            attend(rows.clone().requires_grad_())
