"""Attention of few columns over bf16 pages: the softmax's weights lose nothing that 32 bits hold but what the header states, where
values cancel and where they are large."""
import math

import pytest
import torch

import cache_reference as ref
import paper_2107_03474_amd as lram
from layer_reference import E, HALF

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16 = torch.bfloat16
TWO_PARTS = 2.0 ** -15  # a weight as two numbers of 8 bits, the first cut (2^-7), the second rounded (2^-8 of that)


def _cache(g, used, kv, dim, page, values):
    each = [-(-n // page) for n in used]
    keys = lram.paged_keys(sum(each), kv, dim, page, BF16, True)
    for t in keys:
        t.zero_()
    table = lram.page_table(len(used), max(each))
    pages = torch.randperm(sum(each), generator=g, device=DEV).to(torch.int32).split(each)
    for b, n in enumerate(each):
        table.table[b, :n] = pages[b]
    n = torch.tensor(used, dtype=torch.int32, device=DEV)
    table.used.copy_(n)
    table.seen.copy_(n)
    store = ref.Store(keys)
    for b, n in enumerate(used):
        p, s = store.places(table.table[b], n)
        store.k[p, s] = torch.randn((n, kv, dim), generator=g, device=DEV).to(BF16)
        store.v[p, s] = values(torch.randn((n, kv, dim), generator=g, device=DEV)).to(BF16)
        store.position[p, s] = torch.arange(n, dtype=torch.int32, device=DEV)[:, None].expand(n, kv)
    store.write()
    return keys, table


FEW = [
    # new rows, used keys, heads, kv_heads, dim, page
    ([1], [1], 8, 8, 64, 32),
    ([1], [777], 8, 8, 64, 32),
    ([1] * 4, [33, 4000, 256, 1100], 32, 8, 128, 64),
    ([1], [30011], 4, 1, 128, 256),
    ([2, 4, 1], [600, 70, 45], 4, 1, 32, 32),
    ([1, 1], [300, 2500], 16, 1, 64, 128),
]


@pytest.mark.parametrize("what", ["cancel", "offset"])
@pytest.mark.parametrize("weigh", [False, True])
@pytest.mark.parametrize("new,used,heads,kv,dim,page", FEW)
def test_weights_are_not_rounded_to_eight_bits(new, used, heads, kv, dim, page, weigh, what):
    """cancel: values of either sign, which leave a result far below their sum of sizes; offset: results next to 0 of values that
    are +-1 alone."""
    g = torch.Generator(device=DEV)
    g.manual_seed(sum(used) + dim)
    keys, table = _cache(g, used, kv, dim, page, (lambda x: x * 100) if what == "cancel" else torch.sign)
    q = torch.randn((sum(new), heads, dim), generator=g, device=DEV).to(BF16)
    seqs = lram.pack(new)._replace(max_q=max(new), max_k=max(used))
    start, scale = seqs.start_q.tolist(), 1 / math.sqrt(dim)
    store = ref.Store(keys)
    want, bound = ref.attention(store, q, table.table, used, used, start, scale)[0]["out"]
    # the same bound with the weights' own rounding in place of one to 8 bits
    sizes = ref.Store(keys)
    sizes.v = store.v.abs()
    size = ref.attention(sizes, q, table.table, used, used, start, scale)[0]["out"][0]
    out = lram.paged_attention(q, keys, table, seqs, scale, weigh=weigh)
    ref.check(out, (want, bound - (HALF[BF16] - TWO_PARTS - 2 * E) * size))


def test_infinite_values_stay_infinite():
    """A key that is met and has an infinite value: the result is that infinity, also where the weight is a power of 2."""
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    keys, table = _cache(g, [4, 100], 1, 32, 32, lambda x: x)
    store = ref.Store(keys)
    for b, n in enumerate((4, 100)):
        p, s = store.places(table.table[b], n)
        if b == 0:
            store.k[p, s] = 0  # four weights of 1/4
        store.v[p[1], s[1], 0, :2] = torch.tensor([math.inf, -math.inf], dtype=BF16, device=DEV)
    store.write()
    q = torch.randn((2, 2, 32), generator=g, device=DEV).to(BF16)
    out = lram.paged_attention(q, keys, table, lram.pack([1, 1])._replace(max_k=100))
    assert (out[:, :, 0] == math.inf).all() and (out[:, :, 1] == -math.inf).all() and torch.isfinite(out[:, :, 2:]).all()
