"""Append of many rows, where a wave takes several heads of a tile, against the same rows in small batches, where it takes one."""
import math

import pytest
import torch

import paper_2107_03474_amd as lram

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _bits(t):
    return t.contiguous().view(torch.int16 if t.dtype is BF16 else torch.int32)


FILLS = [
    # new rows of each sequence, keys before, heads, kv_heads, dim, page, pairs, interleaved, dtype; heads of a wave
    ([9001, 0, 33, 1, 7000, 31, 64, 3881], [5, 7, 0, 31, 64, 1, 100, 0], 8, 8, 128, 64, 64, False, BF16),  # 2
    ([20011], [17], 8, 8, 64, 256, 0, False, BF16),                                                     # 2, nothing turns
    ([12345, 5, 25702], [0, 90, 13], 7, 7, 64, 32, 30, True, BF16),                                       # 4, then 3
    ([27003], [2], 10, 5, 32, 128, 13, False, F32),                                                     # 2, 2, then 1
    ([15000, 1, 999, 9003, 2022], [33, 0, 0, 8, 1], 10, 5, 64, 32, 32, False, F32),
    ([70003, 31], [1, 3], 8, 8, 32, 64, 16, True, BF16),                                                 # 8
]


@pytest.mark.parametrize("new,before,heads,kv,dim,page,pairs,interleaved,dtype", FILLS)
def test_many_rows_are_stored_as_few(new, before, heads, kv, dim, page, pairs, interleaved, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(sum(new))
    lead, tail = 2, 3
    rows = lead + sum(new) + tail
    x = torch.randn((rows, (heads + 2 * kv) * dim), generator=g, device=DEV).to(dtype)
    q = x[:, :heads * dim].unflatten(1, (heads, dim))
    k, v = (x[:, (heads + i * kv) * dim:(heads + (i + 1) * kv) * dim].unflatten(1, (kv, dim)) for i in (0, 1))
    given = torch.rand((rows, kv), generator=g, device=DEV)
    plan = lram.rotary_plan(2 * pairs, interleaved=interleaved)._replace(magnitude=1.1) if pairs else None
    each = [-(-(m + n) // page) for m, n in zip(before, new)]
    order = torch.randperm(sum(each) + 1, generator=g, device=DEV).to(torch.int32).split(each + [1])
    start = [lead]
    for n in new:
        start.append(start[-1] + n)

    def filled(batch):
        keys = lram.paged_keys(sum(each) + 1, kv, dim, page, dtype, True)
        for t in keys:
            t.fill_(-7 if t.dtype is torch.int32 else math.nan)
        table = lram.page_table(len(new), max(each))
        for b, n in enumerate(each):
            table.table[b, :n] = order[b]
        table.used.copy_(_ints(before))
        table.seen.copy_(_ints(before) + 5)  # keys were lost
        turned = []
        for r in range(0, rows, batch):
            n = min(batch, rows - r)
            at = [min(max(s - r, 0), n) for s in start]
            longest = max(b - a for a, b in zip(at, at[1:]))
            seqs = lram.Packed(_ints(at), _ints(at), longest, 1)
            lram.paged_extend(table, seqs)
            y = lram.paged_append(k[r:r + n], v[r:r + n], keys, table, seqs, q=q[r:r + n], rotary=plan, weight=given[r:r + n])
            turned.append(y)
        assert table.used.tolist() == [m + n for m, n in zip(before, new)]
        return keys, torch.cat(turned)

    got, got_q = filled(rows)
    want, want_q = filled(4003)  # 4,003 / 16 tiles of 8 heads: a wave takes one
    for name, a, b in zip(got._fields, got, want):
        assert torch.equal(_bits(a), _bits(b)), name
    assert torch.equal(_bits(got_q), _bits(want_q))
