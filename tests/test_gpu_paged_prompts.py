"""Prompts and pieces of them through pages, alone and beside single tokens, against the 64-bit form with its derived bounds; the
layer served from bf16 pages; append where no length fits."""
import math

import pytest
import torch

import cache_reference as ref
import paper_2107_03474_amd as lram
from layer_reference import E
from paper_2107_03474_amd.memory_block import MemoryBlock

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _bits(t):
    return t.contiguous().view(torch.uint8)


def _filled(g, used, kv, dim, page, dtype, seen=None):
    """A cache of so many keys; where tokens were lost, in any order.  Slots past the keys hold NaN."""
    each = [-(-n // page) for n in used]
    keys = lram.paged_keys(sum(each), kv, dim, page, dtype, True)
    for t in keys:
        t.fill_(-7 if t.dtype is torch.int32 else math.nan)
    table = lram.page_table(len(used), max(each))
    order = torch.randperm(sum(each), generator=g, device=DEV).to(torch.int32).split(each)
    for b, n in enumerate(each):
        table.table[b, :n] = order[b]
    table.used.copy_(_ints(used))
    table.seen.copy_(_ints(seen or used))
    store = ref.Store(keys)
    for b, n in enumerate(used):
        p, s = store.places(table.table[b], n)
        for t in (store.k, store.v):
            t[p, s] = torch.randn((n, kv, dim), generator=g, device=DEV).to(dtype)
        at = torch.arange(n, device=DEV).expand(kv, n) if not seen else torch.rand((kv, seen[b]), generator=g, device=DEV).argsort(1)[:, :n]
        store.position[p, s] = at.t().to(torch.int32)
        store.weight[p, s] = torch.rand((n, kv), generator=g, device=DEV)
    store.write()
    return keys, table


PROMPTS = [
    # new rows, used keys, tokens had where some were lost, heads, kv_heads, dim, page, dtype
    ([300, 511], [300, 511], None, 8, 8, 128, 256, BF16),
    ([1000], [1000], None, 8, 2, 64, 64, BF16),
    ([777, 1, 260], [777, 900, 1500], None, 6, 3, 32, 32, F32),
    ([513], [513], None, 4, 4, 128, 128, F32),
    # a piece of a prompt beside single tokens over caches of many pieces
    ([256, 1], [256, 20000], None, 8, 2, 128, 64, BF16),
    ([1, 300, 1, 33], [9001, 5000, 64, 33], None, 8, 8, 64, 32, BF16),
    ([1, 200], [12345, 700], None, 8, 4, 64, 128, F32),
    ([1, 256, 2], [6000, 4000, 3000], [9000, 4001, 50000], 16, 2, 64, 64, BF16),
]


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("new,used,seen,heads,kv,dim,page,dtype", PROMPTS)
def test_prompts_and_pieces(new, used, seen, heads, kv, dim, page, dtype, bias):
    g = _gen(sum(used) + heads + bias)
    keys, table = _filled(g, used, kv, dim, page, dtype, seen)
    q = torch.randn((sum(new), heads, dim), generator=g, device=DEV).to(dtype) * 2
    rel = None
    if bias:
        rel = lram.RelativeBias(torch.randn((heads, 32), generator=g, device=DEV).to(dtype), lram.relative_buckets(32, 100, both=False))
    seqs = lram.pack(new)._replace(max_k=max(used))
    store, before, scale = ref.Store(keys), keys.weight.clone(), 0.8 / math.sqrt(dim)
    want, more, bound = ref.attention(store, q, table.table, used, seen or used, seqs.start_q.tolist(), scale,
                                      rel.weight if rel else None, rel.bucket if rel else None)
    out = lram.paged_attention(q, keys, table, seqs, scale, rel)
    ref.check(out, want["out"])
    assert torch.equal(_bits(keys.weight), _bits(before))
    assert torch.equal(lram.paged_attention(q, keys, table, seqs, scale, rel, weigh=True), out)
    got, met = ref.Store(keys).weight, bound > 0
    total = store.weight.double() + more
    assert ((got.double() - total).abs() <= bound + 2 * E * total.abs())[met].all()
    assert torch.equal(_bits(got[~met]), _bits(store.weight[~met]))


@pytest.mark.parametrize("rotary", [False, True])
def test_a_layer_served_from_bf16_pages(rotary):
    """Prompts, pieces and single tokens: what attention hands on, against the 64-bit form over the pages as they then are."""
    torch.manual_seed(5)
    plan = lram.rotary_plan(32, scaling="parts", factor=4.0, length=100) if rotary else None
    block = MemoryBlock(256, 4, (4,) * 8, 2, True, buckets=16, reach=20, dtype=BF16, rotary=plan).eval()
    if not rotary:
        with torch.no_grad():
            block.bias.normal_()
    cache = lram.PagedCache(3, 30, 2, 64, page=32, dtype=BF16, weigh=True)
    handed = []
    block.proj.register_forward_pre_hook(lambda m, a: handed.append(a[0].unflatten(1, (4, 64))))
    for step in ([300, 33, 1], [1, 100, 1], [1, 1, 1], [0, 1, 40], [1, 1, 1]):
        x = torch.randn((sum(step), 256), device=DEV).to(BF16)
        seqs = cache.extend(lram.pack(step), step)
        old = ref.Store(cache.keys[0]).weight
        y = block.serve(x, seqs, cache)
        assert y.dtype is BF16 and y.shape == x.shape and torch.isfinite(y).all()
        with torch.no_grad():
            q, k, v = block._heads(x)
        used, start = cache.table.used.tolist(), seqs.start_q.tolist()
        if rotary:
            at = lram.packed_positions(seqs, sum(step), cache.table.seen - _ints(step))
            q, k = lram.rotary_forward(q, k, at, plan)
        store = ref.Store(cache.keys[0])
        for b, n in enumerate(step):
            p, s = (t[used[b] - n:] for t in store.places(cache.table.table[b], used[b]))
            assert torch.equal(store.k[p, s], k[start[b]:start[b + 1]]) and torch.equal(store.v[p, s], v[start[b]:start[b + 1]])
            old[p, s] = 0
        want, more, bound = ref.attention(store, q, cache.table.table, used, used, start, 1 / 8, None if rotary else block.bias.detach(),
                                          None if rotary else block.bucket)
        ref.check(handed.pop(), want["out"], step)
        for b, n in enumerate(used):
            p, s = store.places(cache.table.table[b], n)
            total = old[p, s].double() + more[p, s]
            assert ((store.weight[p, s].double() - total).abs() <= bound[p, s] + 2 * E * total.abs()).all()


@pytest.mark.parametrize("used", [-5, 0, -(1 << 31)])
def test_append_where_no_length_fits(used):
    """Lengths below the new rows' number, which were never counted: nothing of the pool changes."""
    g = _gen(6)
    keys, table = _filled(g, [60, 20], 2, 64, 32, BF16)
    before = [_bits(t).clone() for t in keys]
    k, v = (torch.randn((39, 2, 64), generator=g, device=DEV).to(BF16) for _ in range(2))
    table.used.fill_(used)
    lram.paged_append(k, v, keys, table, lram.pack([9, 30]))
    assert all(torch.equal(_bits(a), b) for a, b in zip(keys, before))
