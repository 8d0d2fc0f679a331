"""The layer around the memory with rotary positions, and served from pages: training, prompts, pieces and single tokens."""
import math

import pytest
import torch

import cache_reference as ref
import paper_2107_03474_amd as lram
from paper_2107_03474_amd.memory_block import KeyValueCache, MemoryBlock

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _block(rotary, seed, causal=True):
    torch.manual_seed(seed)
    plan = lram.rotary_plan(24, interleaved=True, scaling="linear", factor=2.0) if rotary else None
    block = MemoryBlock(128, 4, (4,) * 8, 2, causal, buckets=16, reach=20, table_dtype=torch.float32, rotary=plan).eval()
    with torch.no_grad():
        for w, b in zip(block.norm_w, block.norm_b):
            w.add_(torch.randn_like(w) * 0.1)
            b.add_(torch.randn_like(b) * 0.1)
        if not rotary:
            block.bias.normal_()
    return block


def test_training_with_a_rotation():
    """The attention's result and gradients of the layer's input, against plain products in 64 bits."""
    block = _block(True, 1, causal=False)
    lengths = [5, 1, 17]
    x = torch.randn((sum(lengths), 128), device=DEV, requires_grad=True)
    seqs = lram.pack(lengths)
    seen = []
    block.proj.register_forward_pre_hook(lambda m, a: seen.append(a[0]))
    block(x, seqs)
    g = torch.randn_like(seen[0])
    got, = torch.autograd.grad(seen[0], x, g)
    at = lram.packed_positions(seqs, sum(lengths))
    assert at.tolist() == [i for n in lengths for i in range(n)]
    x64 = x.detach().double().requires_grad_()
    y = x64 @ block.qkv.weight.double().t() + block.qkv.bias.double()
    q, k, v = y[:, :128].unflatten(1, (4, 32)), y[:, 128:192].unflatten(1, (2, 32)), y[:, 192:].unflatten(1, (2, 32))
    a = ref.angles(block.turns, at)[:, None]

    def turned(t):
        z = torch.view_as_complex(t[..., :24].unflatten(-1, (12, 2)).contiguous()) * torch.polar(torch.ones_like(a), a)
        return torch.cat([torch.view_as_real(z).flatten(-2), t[..., 24:]], -1)

    q, k = turned(q), turned(k)
    out, row = [], 0
    for n in lengths:
        qs, ks, vs = (t[row:row + n].transpose(0, 1) for t in (q, k.repeat_interleave(2, 1), v.repeat_interleave(2, 1)))
        out.append((torch.softmax(qs @ ks.transpose(1, 2) / math.sqrt(32), 2) @ vs).transpose(0, 1).flatten(1))
        row += n
    out = torch.cat(out)
    want, = torch.autograd.grad(out, x64, g.double())
    # fp32 products of 128 terms through the projection, the scores and back
    assert (seen[0].double() - out).abs().max() < 1e-5
    assert (got.double() - want).abs().max() < 1e-4
    block.zero_grad()
    block(x, seqs, at).square().sum().backward()
    assert all(p.grad is not None for p in block.parameters())
    assert "bias" not in dict(block.named_parameters()) and "turns" in block.state_dict()


@pytest.mark.parametrize("rotary", [False, True])
def test_served_from_pages_as_from_rows_of_their_own(rotary):
    """The same texts, whole, in pieces and token by token, from a contiguous cache, from pages, and at once."""
    blocks = [_block(rotary, s) for s in (2, 3)]
    lengths = [70, 33, 1]
    texts = [torch.randn((n, 128), device=DEV) for n in lengths]
    want = torch.cat(texts)
    seqs = lram.pack(lengths)
    for b in blocks:
        with torch.no_grad():
            want = b(want, seqs)
    want = want.split(lengths)
    pages = lram.PagedCache(3, 12, 2, 32, page=32, capacity=96, layers=2, dtype=torch.float32)
    rows = [KeyValueCache(3, 96, 2, 32, torch.float32) for _ in blocks]
    done = [0, 0, 0]
    for step in ([40, 33, 0], [20, 0, 1], [1, 0, 0], [1, 0, 0], [8, 0, 0]):
        x = torch.cat([t[d:d + n] for t, d, n in zip(texts, done, step)])
        plan = lram.pack(step)
        y, z = x, x
        seqs = pages.extend(plan, step)
        for i, b in enumerate(blocks):
            y = b.serve(y, seqs, pages, i)
            z = b.serve(z, plan, rows[i])
        at = 0
        for t, (d, n) in enumerate(zip(done, step)):
            # the same rows in other batches: the projections may sum in another order
            assert n == 0 or (y[at:at + n] - want[t][d:d + n]).abs().max() < 5e-4
            assert n == 0 or (z[at:at + n] - want[t][d:d + n]).abs().max() < 5e-4
            at += n
        done = [d + n for d, n in zip(done, step)]
    assert pages.refresh() == lengths and rows[0].used.tolist() == lengths
    with pytest.raises(ValueError, match="capacity"):
        pages.extend(lram.pack([30, 1, 1]), [30, 1, 1])


def test_served_under_a_budget():
    """A text that stays under the budget is served as without one; a longer one goes on from the keys that stayed."""
    block = _block(True, 4)
    cache = lram.PagedCache(2, 8, 2, 32, page=32, dtype=torch.float32, weigh=True)
    free = lram.PagedCache(2, 8, 2, 32, page=32, dtype=torch.float32)
    x = torch.randn((60, 128), device=DEV)
    for step in ([40, 10], [1, 1], [1, 1], [1, 1], [1, 1], [0, 1]):
        part = x[:sum(step)]
        x = x.roll(-sum(step), 0)
        y = block.serve(part, cache.extend(lram.pack(step), step), cache)
        z = block.serve(part, free.extend(lram.pack(step), step), free)
        assert (y[step[0]:] - z[step[0]:]).abs().max() < 5e-4 and torch.isfinite(y).all()
        cache.evict(32, 8)
        assert cache.table.used.tolist()[0] <= 32
    assert cache.table.used.tolist() == [32, 15] and cache.table.seen.tolist() == [44, 15]
    at = lram.paged_read(cache.keys[0], cache.table, 0)[2]
    for h in range(2):  # the newest are all there, and no key twice
        kept = at[:, h].tolist()
        assert set(range(36, 44)) <= set(kept) and len(set(kept)) == 32


def test_refusals():
    with pytest.raises(ValueError, match="pairs"):
        MemoryBlock(128, 4, (4,) * 8, rotary=lram.rotary_plan(34))
    block = _block(True, 5, causal=False)
    with pytest.raises(ValueError, match="causal"):
        block.serve(torch.zeros((1, 128), device=DEV), lram.pack([1]), lram.PagedCache(1, 2, 2, 32, 32, dtype=torch.float32))
