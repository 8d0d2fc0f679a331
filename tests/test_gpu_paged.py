"""The cache in pages, attention over it and eviction from it against plain 64-bit forms, with bounds from the arithmetic that the
header states."""
import math

import pytest
import torch

import cache_reference as ref
import paper_2107_03474_amd as lram
from layer_reference import E

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _plan(new, before=0, max_q=None, max_k=1):
    seqs = lram.pack(new)
    return seqs._replace(start_q=seqs.start_q + before, max_q=max(new, default=0) if max_q is None else max_q, max_k=max_k)


def _cache(g, used, kv, dim, page, dtype, spare=2, seen=None, weigh=True, width=None, poison=math.nan, more=None):
    """A cache whose sequences use so many keys, pages in any order, with room for more: (keys, table).  Slots past the keys hold
    NaN."""
    each = [-(-(n + m) // page) + 1 for n, m in zip(used, more or [0] * len(used))]
    total = sum(each) + spare
    keys = lram.paged_keys(total, kv, dim, page, dtype, weigh)
    keys.k.fill_(poison)
    keys.v.fill_(poison)
    keys.position.fill_(-7)
    if weigh:
        keys.weight.fill_(poison)
    table = lram.page_table(len(used), width or max(each, default=1))
    order = torch.randperm(total, generator=g, device=DEV).tolist()
    for b, n in enumerate(each):
        n = min(n, table.table.shape[1])
        table.table[b, :n] = _ints(order[:n])
        order = order[n:]
    table.used.copy_(_ints(used))
    table.seen.copy_(_ints(used if seen is None else seen))
    store = ref.Store(keys)
    for b, n in enumerate(used):
        p, s = store.places(table.table[b], n)
        store.k[p, s] = torch.randn((len(p), kv, dim), generator=g, device=DEV).to(dtype)
        store.v[p, s] = torch.randn((len(p), kv, dim), generator=g, device=DEV).to(dtype)
        most = n if seen is None else seen[b]
        at = torch.rand((kv, most), generator=g, device=DEV).argsort(1)[:, :n].t() if seen else torch.arange(n, device=DEV)[:, None].expand(n, kv)
        store.position[p, s] = at[:len(p)].to(torch.int32)
        if weigh:
            store.weight[p, s] = torch.rand((len(p), kv), generator=g, device=DEV)
    store.write()
    return keys, table


def _same(a, b):
    """Equal bits."""
    return a.shape == b.shape and torch.equal(a.flatten().view(torch.uint8), b.flatten().view(torch.uint8))


def _unchanged(keys):
    return [None if t is None else t.clone() for t in keys]


def test_the_layout_is_the_headers():
    """k and v of PagedKeys, by its own docstring, against the header's formula, and back."""
    for dtype in (BF16, F32):
        keys = lram.paged_keys(3, 2, 64, 64, dtype, True)
        e = 16 // keys.k.element_size()
        keys.k.copy_(torch.randn(keys.k.shape, device=DEV))
        keys.v.copy_(torch.randn(keys.v.shape, device=DEV))
        store = ref.Store(keys)
        for t, d in ((0, 0), (1, 5), (17, 63), (33, 30), (63, 17), (44, 8)):
            assert torch.equal(store.k[:, t, :, d], keys.k[:, :, t // 16, d // e, t % 16, d % e])
            assert torch.equal(store.v[:, t, :, d], keys.v[:, :, t // (4 * e), d // 16, t % 16 // 4, d % 16,
                                                           t % (4 * e) // 16 * 4 + t % 4])
        before = _unchanged(keys)
        store.write()
        assert _same(before[0], keys.k) and _same(before[1], keys.v)


# ---------------------------------------------------------------------------
# Append.

APPEND = [
    # new rows of each sequence, keys before, heads, kv_heads, dim, page, pairs, interleaved, dtype
    ([1], [0], 8, 8, 64, 32, 32, False, BF16),
    ([1, 1, 1, 1], [0, 31, 32, 777], 32, 8, 128, 64, 64, False, BF16),
    ([0, 5, 33, 70, 1], [3, 30, 100, 1, 63], 4, 2, 32, 32, 16, True, BF16),
    ([200, 0, 3], [0, 0, 250], 6, 2, 64, 256, 17, False, F32),
    ([31, 64, 1], [1, 0, 64], 3, 3, 128, 128, 5, True, F32),
    ([40, 9], [10, 0], 4, 1, 64, 64, 0, False, BF16),
    ([1, 0, 2] * 100, [7, 40, 31] * 100, 2, 1, 32, 32, 16, False, BF16),  # more sequences than a wave has lanes
    ([70, 1] * 40, [0, 5] * 40, 4, 2, 64, 32, 9, True, F32),
]


@pytest.mark.parametrize("understated", [False, True])
@pytest.mark.parametrize("new,before,heads,kv,dim,page,pairs,interleaved,dtype", APPEND)
def test_append(new, before, heads, kv, dim, page, pairs, interleaved, dtype, understated):
    g = _gen(len(new) + dim)
    seen = [n + 1000 * b for b, n in enumerate(before)]  # some have lost keys
    keys, table = _cache(g, before, kv, dim, page, dtype, seen=[max(s, 1) for s in seen], more=new)
    lead, tail = 2, 3
    rows = sum(new) + lead + tail
    x = torch.randn((rows, (heads + 2 * kv) * dim), generator=g, device=DEV).to(dtype)
    q = x[:, :heads * dim].unflatten(1, (heads, dim))
    k, v = (x[:, (heads + i * kv) * dim:(heads + (i + 1) * kv) * dim].unflatten(1, (kv, dim)) for i in (0, 1))
    given = torch.rand((rows, kv), generator=g, device=DEV)
    plan = lram.rotary_plan(2 * pairs, interleaved=interleaved)._replace(magnitude=1.1) if pairs else None
    seqs = _plan(new, lead, 1 if understated else None)
    want = ref.Store(keys)
    start = [max(s, 1) for s in seen]
    lram.paged_extend(table, seqs)
    assert table.used.tolist() == [a + b for a, b in zip(before, new)]
    assert table.seen.tolist() == [a + b for a, b in zip(start, new)]
    got_q = lram.paged_append(k, v, keys, table, seqs, q=q, rotary=plan, weight=given)
    got = ref.Store(keys)
    at = torch.zeros(rows, dtype=torch.int32, device=DEV)
    row = lead
    for b, n in enumerate(new):
        at[row:row + n] = torch.arange(n, dtype=torch.int32, device=DEV) + start[b]
        p, s = (t[before[b]:] for t in want.places(table.table[b], before[b] + n))
        if plan is not None and n:
            ref.check(got.k[p, s], ref.rotated(k[row:row + n], at[row:row + n], plan.turns, interleaved, 1.1))
            want.k[p, s] = got.k[p, s]
        else:
            want.k[p, s] = k[row:row + n]
        want.v[p, s] = v[row:row + n]
        want.position[p, s] = at[row:row + n, None].expand(n, kv)
        want.weight[p, s] = given[row:row + n]
        row += n
    for name in ("k", "v", "position", "weight"):
        assert _same(getattr(got, name), getattr(want, name)), name  # and nothing else has changed
    if plan is None:
        assert got_q is q
    else:
        ref.check(got_q, ref.rotated(q, at, plan.turns, interleaved, 1.1))
        assert lram.paged_append(k, v, keys, table, seqs, rotary=plan) is None  # again, without q and weights
        assert _same(ref.Store(keys).k, want.k)
        for b, n in enumerate(new):
            p, s = (t[before[b]:] for t in want.places(table.table[b], before[b] + n))
            assert (ref.Store(keys).weight[p, s] == 0).all()


def test_append_leaves_out_what_has_no_place():
    """Rows past the capacity, rows of pages that are none, and lengths that were never counted."""
    g = _gen(5)
    keys, table = _cache(g, [60, 20, 40, 0], 2, 64, 32, BF16, width=2)
    table.table[1] = _ints([-1, 10000])
    table.table[2, 1] = -1
    new = [9, 30, 8, 3]
    k, v = (torch.randn((sum(new), 2, 64), generator=g, device=DEV).to(BF16) for _ in range(2))
    seqs = _plan(new)
    before = _unchanged(keys)
    want = ref.Store(keys)
    lram.paged_extend(table, seqs)
    table.used[3] = 2  # fewer than its three new rows: the first has no slot
    lram.paged_append(k, v, keys, table, seqs)
    p, s = want.places(table.table[0], 64)
    want.k[p[60:], s[60:]], want.v[p[60:], s[60:]] = k[:4], v[:4]
    want.position[p[60:], s[60:]] = torch.arange(60, 64, device=DEV, dtype=torch.int32)[:, None]
    want.weight[p[60:], s[60:]] = 0
    p, s = want.places(table.table[3], 2)
    want.k[p, s], want.v[p, s] = k[-2:], v[-2:]
    want.position[p, s] = _ints([1, 2])[:, None].expand(2, 2)
    want.weight[p, s] = 0
    got = ref.Store(keys)
    for name in ("k", "v", "position", "weight"):
        assert _same(getattr(got, name), getattr(want, name)), name
    table.used.fill_(-5)
    lram.paged_append(k, v, keys, table, seqs)
    assert _same(keys.k, ref.Store(keys).keys.k) and _same(ref.Store(keys).v, want.v) and not _same(before[0], keys.k)


# ---------------------------------------------------------------------------
# Attention.

ATTEND = [
    # new rows, used keys, heads, kv_heads, dim, page, dtype
    ([1], [1], 8, 8, 64, 32, BF16),
    ([1], [777], 8, 8, 64, 32, BF16),
    ([1] * 5, [1, 31, 33, 4000, 0], 32, 8, 128, 64, BF16),
    ([1, 3, 0, 2, 7], [129, 1000, 5, 2500, 7], 8, 4, 64, 32, F32),
    ([1, 16, 5], [3000, 16, 511], 16, 1, 128, 256, F32),
    ([40, 1, 100], [40, 600, 1500], 6, 2, 32, 64, BF16),
    ([17, 33], [17, 900], 8, 2, 128, 128, BF16),
    ([2, 1], [600, 70], 64, 1, 32, 32, BF16),
    ([1] * 70, list(range(70)), 4, 2, 32, 32, F32),
    ([30], [513], 3, 3, 32, 64, F32),
    ([1], [1100], 32, 8, 128, 64, BF16),  # the least pieces
    ([3], [1501], 8, 4, 64, 32, F32),
    ([1] * 136, [600] + [7 * i % 41 for i in range(135)], 4, 4, 128, 64, BF16),   # heads of sequences that fill the card
    ([1] * 136, [2100] + [7 * i % 41 for i in range(135)], 4, 4, 128, 64, BF16),  # and keys past one piece
]


@pytest.mark.parametrize("evicted", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("new,used,heads,kv,dim,page,dtype", ATTEND)
def test_attention(new, used, heads, kv, dim, page, dtype, bias, evicted):
    g = _gen(sum(used) + bias)
    seen = [2 * n + 50 for n in used] if evicted else None
    keys, table = _cache(g, used, kv, dim, page, dtype, seen=seen)
    if evicted and len(used) > 1:  # a page that is none: its keys are not met
        table.table[-1, 0] = -1 if bias else 10 ** 6
    lead, tail = 2, 1
    rows = sum(new) + lead + tail
    q = torch.randn((rows, heads * dim + 16), generator=g, device=DEV).to(dtype)[:, :heads * dim].unflatten(1, (heads, dim)) * 2
    q = q.as_strided(q.shape, (heads * dim, dim, 1)) if q.is_contiguous() else q
    rel = None
    if bias:
        reach = min(128, (4096 // (heads // kv) - 193) // 2) if heads // kv <= 16 else 0
        if heads // kv > 16:
            pytest.skip("a bias holds at most 4096 / 193 heads of a group")
        w = torch.randn((heads, 32), generator=g, device=DEV).to(dtype)
        w[0, 3] = -math.inf
        rel = lram.RelativeBias(w, lram.relative_buckets(32, max(reach, 16), both=False) if reach >= 16 else _ints([3] * (2 * reach + 1)))
    seqs = _plan(new, lead, max_k=max(used, default=0))
    start = seqs.start_q.tolist()
    scale = 0.7 / math.sqrt(dim)
    before, store = _unchanged(keys), ref.Store(keys)
    want, more, more_bound = ref.attention(store, q, table.table, used, seen or used, start, scale, rel.weight if rel else None,
                                           rel.bucket if rel else None)
    out = lram.paged_attention(q, keys, table, seqs, scale, rel)
    ref.check(out, want["out"])
    for a, b in zip(keys, before):
        assert _same(a, b)
    weighed = lram.paged_attention(q, keys, table, seqs, scale, rel, weigh=True)
    assert _same(weighed, out)
    got = ref.Store(keys).weight
    met = more_bound > 0
    total = store.weight.double() + more
    assert ((got.double() - total).abs() <= more_bound + 2 * E * total.abs())[met].all()
    assert _same(got[~met], store.weight[~met])
    for a, b in zip(keys[:3], before[:3]):
        assert _same(a, b)
    first = keys.weight.clone()
    keys.weight.copy_(before[3])
    for wrong in ((1, 1), (1, 10 ** 9), (10 ** 6, 1), (0, 0)):  # expectations that say little: other divisions of the work
        s = seqs._replace(max_q=wrong[0], max_k=wrong[1])
        ref.check(lram.paged_attention(q, keys, table, s, scale, rel, weigh=True), want["out"])
        got = ref.Store(keys).weight
        assert ((got.double() - total).abs() <= more_bound + 2 * E * total.abs())[met].all() and _same(got[~met], store.weight[~met])
        keys.weight.copy_(before[3])
    lram.paged_attention(q, keys, table, seqs, scale, rel, weigh=True)
    assert _same(keys.weight, first)  # the same bits on every call


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("cols", [1, 4])
def test_rows_that_the_tensor_does_not_hold(cols, dtype):
    """Starts past q's end: the rows that are there, in their places, and weights of these alone."""
    g = _gen(21)
    new, used, heads = [5, 3, 4], [300, 200, 40], cols
    keys, table = _cache(g, used, 1, 64, 32, dtype)
    q = torch.randn((6, heads, 64), generator=g, device=DEV).to(dtype)  # 5 rows, one of three, and none of four
    seqs = _plan(new, max_k=300)
    store = ref.Store(keys)
    want, more, bound = ref.attention(store, q, table.table, used, [300, 198, 36], [0, 5, 6, 6], 0.125)
    out = lram.paged_attention(q, keys, table, seqs, weigh=True)
    ref.check(out, want["out"])
    got, met = ref.Store(keys).weight, bound > 0
    total = store.weight.double() + more
    assert ((got.double() - total).abs() <= bound + 2 * E * total.abs())[met].all()
    assert _same(got[~met], store.weight[~met])
    k, v = (torch.randn((6, 1, 64), generator=g, device=DEV).to(dtype) for _ in range(2))
    lram.paged_append(k, v, keys, table, seqs)
    after = ref.Store(keys)
    p, s = store.places(table.table[0], 300)
    store.k[p[295:], s[295:]] = k[:5]
    p, s = store.places(table.table[1], 200)
    store.k[p[197], s[197]] = k[5]
    assert _same(after.k, store.k)


def test_gradients_are_refused():
    g = _gen(22)
    keys, table = _cache(g, [10], 2, 64, 32, F32)
    q = torch.randn((1, 2, 64), device=DEV, requires_grad=True)
    for call in (lambda: lram.paged_attention(q, keys, table, _plan([1])), lambda: lram.paged_append(q, q, keys, table, _plan([1]))):
        with pytest.raises(lram.LramError, match="no gradients"):
            call()
        with torch.no_grad():
            call()


def test_no_sequences_and_no_pages():
    g = _gen(8)
    keys, table = _cache(g, [], 2, 64, 32, BF16)
    q = torch.randn((3, 4, 64), device=DEV).to(BF16)
    seqs = _plan([])
    assert (lram.paged_attention(q, keys, table, seqs) == 0).all()
    lram.paged_extend(table, seqs)
    lram.paged_append(q[:, :2], q[:, 2:], keys, table, seqs)
    lram.paged_evict(keys, table, 3, 1)
    none, empty = lram.paged_keys(0, 2, 64, 32, BF16, True), lram.page_table(2, 0)
    seqs = _plan([1, 2])
    lram.paged_extend(empty, seqs)
    lram.paged_append(q[:, :2], q[:, 2:], none, empty, seqs)
    assert (lram.paged_attention(q, none, empty, seqs, weigh=True) == 0).all()
    lram.paged_evict(none, empty, 1)
    assert lram.paged_attention(q[:0], keys, table, _plan([])).shape == (0, 4, 64)


def test_values_that_are_not_finite_stay_in_their_sequence():
    g = _gen(9)
    keys, table = _cache(g, [100, 100], 2, 64, 32, BF16)
    store = ref.Store(keys)
    p, s = store.places(table.table[0], 100)
    store.k[p[5], s[5]] = math.nan
    store.v[p[7], s[7]] = math.inf
    store.write()
    q = torch.randn((2, 4, 64), generator=g, device=DEV).to(BF16)
    out = lram.paged_attention(q, keys, table, _plan([1, 1], max_k=100), weigh=True)
    assert torch.isnan(out[0]).all() and torch.isfinite(out[1]).all()
    p, s = store.places(table.table[1], 100)
    assert torch.isfinite(ref.Store(keys).weight[p, s]).all()


@pytest.mark.parametrize("value", [-3e38, 3e38, -1.2e7])
def test_vast_weights(value):
    """Finite weights past any score count alike: the even average of the keys that have them, or nothing beside others."""
    g = _gen(10)
    keys, table = _cache(g, [40], 1, 32, 32, F32)
    q = torch.randn((1, 1, 32), generator=g, device=DEV)
    rel = lram.RelativeBias(torch.full((1, 4), value, device=DEV), _ints([3, 2, 2, 1, 1, 0, 0, 0, 0]))
    store = ref.Store(keys)
    p, s = store.places(table.table[0], 40)
    out = lram.paged_attention(q, keys, table, _plan([1], max_k=40), rel=rel)
    assert (out[0, 0].double() - store.v[p, s, 0].double().mean(0)).abs().max() < 64 * E * 5
    rel.weight[0, 2] = 0.0  # the keys 2 and 3 behind
    out = lram.paged_attention(q, keys, table, _plan([1], max_k=40), rel=rel)
    at = [36, 37] if value < 0 else [i for i in range(40) if i not in (36, 37)]
    z = (store.k[p[at], s[at], 0].double() @ q[0, 0].double()) / math.sqrt(32) if value < 0 else torch.zeros(len(at), device=DEV).double()
    want = torch.softmax(z, 0) @ store.v[p[at], s[at], 0].double()
    assert (out[0, 0].double() - want).abs().max() < 200 * E * 5


def test_keys_past_four_gigabytes():
    """Offsets that pass 32 bits, in bytes and in elements: the last pages of a pool of 2^32 elements and more."""
    pages, kv, dim, page = (1 << 32) // (8 * 128 * 256) + 40, 8, 128, 256
    keys = lram.paged_keys(pages, kv, dim, page, BF16, True)
    assert keys.k.numel() > 1 << 32
    table = lram.page_table(2, 2)
    table.table.copy_(_ints([[pages - 1, 0], [1, pages - 2]]))
    g = _gen(11)
    new = [300, 511]
    k, v = (torch.randn((sum(new), kv, dim), generator=g, device=DEV).to(BF16) for _ in range(2))
    seqs = _plan(new, max_k=511)
    lram.paged_extend(table, seqs)
    lram.paged_append(k, v, keys, table, seqs)
    q = torch.randn((sum(new), kv, dim), generator=g, device=DEV).to(BF16)
    out = lram.paged_attention(q, keys, table, seqs, weigh=True)
    want = lram.attention_forward(q, k, v, lram.pack(new), True)[0]
    assert (out.float() - want.float()).abs().max() < 0.05  # two bf16 results of values up to 5
    for b, n in enumerate(new):
        got = lram.paged_read(keys, table, b)
        at = sum(new[:b])
        assert torch.equal(got[0], k[at:at + n]) and torch.equal(got[1], v[at:at + n])
        assert torch.equal(got[2], torch.arange(n, device=DEV, dtype=torch.int32)[:, None].expand(n, kv))
        assert ((got[3].sum(0) - n).abs() < 1e-2).all()  # each query gives away 1
    lram.paged_evict(keys, table, 200, 10)
    lram.paged_shrink(table, 1 << 40)
    assert table.used.tolist() == new
    lram.paged_shrink(table, 200)
    assert [len(lram.paged_read(keys, table, b)[0]) for b in (0, 1)] == [200, 200]


# ---------------------------------------------------------------------------
# Eviction.

EVICT = [
    # used, seen, budget, recent, kv_heads, dim, page, dtype
    ([33], [33], 32, 0, 1, 32, 32, F32),
    ([2049, 2048, 100, 0, 3000], [9000, 2048, 100, 0, 3000], 2048, 64, 2, 128, 64, BF16),
    ([500, 129, 1], [500, 200, 1], 1, 0, 3, 64, 32, BF16),
    ([500, 129, 1], [700, 200, 1], 1, 1, 3, 64, 32, F32),
    ([1500], [100000], 700, 700, 2, 64, 256, F32),
    ([5000, 1025], [5000, 1025], 513, 100, 2, 32, 128, BF16),
    ([20000, 16390], [50000, 16390], 16385, 100, 1, 32, 256, F32),
    ([17500, 70], [17500, 70], 64, 64, 1, 64, 256, BF16),
]


@pytest.mark.parametrize("kind", ["spread", "equal", "few", "odd"])
@pytest.mark.parametrize("used,seen,budget,recent,kv,dim,page,dtype", EVICT)
def test_evict(used, seen, budget, recent, kv, dim, page, dtype, kind):
    g = _gen(sum(used) + budget)
    keys, table = _cache(g, used, kv, dim, page, dtype, seen=[max(n, 1) for n in seen])
    table.seen.copy_(_ints(seen))
    store = ref.Store(keys)
    w = store.weight
    if kind == "equal":
        w.fill_(0.5)
    elif kind == "few":
        w.copy_((torch.rand(w.shape, generator=g, device=DEV) * 4).floor_() / 4)
    elif kind == "odd":  # what a weight can become: NaN, infinities, zeros of both signs, negative numbers
        pick = torch.tensor([math.nan, math.inf, -math.inf, 0.0, -0.0, -1.5, 1e-42, 3e38], device=DEV)
        w.copy_(pick[torch.randint(0, 8, w.shape, generator=g, device=DEV)])
    store.write()
    want = ref.Store(keys)
    ref.evicted(want, table.table, used, seen, budget, recent)
    lram.paged_evict(keys, table, budget, recent)
    got = ref.Store(keys)
    for name in ("k", "v", "position", "weight"):
        assert _same(getattr(got, name), getattr(want, name)), name
    assert table.used.tolist() == used and table.seen.tolist() == seen
    lram.paged_shrink(table, budget)
    assert table.used.tolist() == [min(n, budget) for n in used]


def test_evict_with_odd_tables():
    """Equal positions, a missing page, and lengths past the table."""
    g = _gen(12)
    keys, table = _cache(g, [100, 100, 64], 2, 32, 32, BF16, width=4)
    store = ref.Store(keys)
    store.position.fill_(3)
    store.weight.copy_((torch.rand(store.weight.shape, generator=g, device=DEV) * 3).floor_())
    store.write()
    want = ref.Store(keys)
    table.table[1, 1] = -1
    table.table[2, 2:] = _ints([-1, 10 ** 6])
    table.used[2] = 10 ** 6
    ref.evicted(want, table.table[:1], [100], [100], 50, 0)
    lram.paged_evict(keys, table, 50, 0)
    got = ref.Store(keys)
    for b in range(1):
        p, s = want.places(table.table[b], 100)
        assert _same(got.k[p, s], want.k[p, s]) and _same(got.weight[p, s], want.weight[p, s])
    for b, n in ((1, 100), (2, 64)):  # what is missing goes first; of the others the largest weights have stayed
        p, s = want.places(table.table[b], n)
        have, low = p >= 0, torch.arange(len(p), device=DEV) < 50
        for h in range(2):
            kept = got.weight[p[have & low], s[have & low], h].sort()[0]
            every = want.weight[p[have], s[have], h].sort()[0]
            assert torch.equal(kept, every[-len(kept):])


# ---------------------------------------------------------------------------
# All together, as a program that serves uses them.

def test_steps_under_a_budget():
    """Prompts, pieces and single tokens, evicting in between, by the wrapper and against the plain forms."""
    g = _gen(13)
    heads, kv, dim, budget, recent = 4, 2, 64, 70, 8
    cache = lram.PagedCache(3, 12, kv, dim, page=32, layers=2, dtype=BF16, weigh=True)
    plan = lram.rotary_plan(32)
    for step, new in enumerate(([50, 1, 90], [1, 1, 1], [1, 40, 1], [0, 33, 1], [1, 1, 1], [1, 1, 0], [1, 1, 1])):
        x = torch.randn((sum(new), heads + 2 * kv, dim), generator=g, device=DEV).to(BF16)
        q, k, v = x[:, :heads], x[:, heads:heads + kv], x[:, heads + kv:]
        seqs = cache.extend(lram.pack(new), new)
        for layer, keys in enumerate(cache.keys):
            turned = lram.paged_append(k, v, keys, cache.table, seqs, q=q, rotary=plan)
            store = ref.Store(keys)
            used, seen = cache.table.used.tolist(), cache.table.seen.tolist()
            want, more, bound = ref.attention(store, turned, cache.table.table, used, seen, seqs.start_q.tolist(), dim ** -0.5)
            ref.check(lram.paged_attention(turned, keys, cache.table, seqs, weigh=True), want["out"], (step, layer))
            got = ref.Store(keys).weight.double()
            for b in range(3):
                p, s = store.places(cache.table.table[b], used[b])
                total = store.weight[p, s].double() + more[p, s]
                assert ((got[p, s] - total).abs() <= bound[p, s] + 2 * E * total).all()
        wants = []
        for keys in cache.keys:
            store = ref.Store(keys)
            ref.evicted(store, cache.table.table, used, seen, budget, recent)
            wants.append(store)
        cache.evict(budget, recent)
        assert cache.table.used.tolist() == [min(n, budget) for n in used] == cache._used
        for keys, want in zip(cache.keys, wants):
            got = ref.Store(keys)
            for b in range(3):
                p, s = want.places(cache.table.table[b], min(used[b], budget))
                assert _same(got.k[p, s], want.k[p, s]) and _same(got.v[p, s], want.v[p, s])
                assert _same(got.position[p, s], want.position[p, s]) and _same(got.weight[p, s], want.weight[p, s])
    cache.trim()
    assert cache.free_pages() == 12 - sum(-(-n // 32) for n in cache.refresh())
    cache.release([0, 1, 2])
    assert cache.free_pages() == 12 and cache.table.seen.tolist() == [0, 0, 0]


def test_a_captured_step_replayed():
    """A whole step in a graph, replayed between eager work, against the same steps without one."""
    g = _gen(14)
    heads, kv, dim, budget = 8, 2, 64, 40
    eager, captured = (lram.PagedCache(3, 9, kv, dim, page=32, dtype=BF16, weigh=True) for _ in range(2))
    plan = lram.rotary_plan(64, interleaved=True)
    x = torch.randn((4, heads + 2 * kv, dim), generator=g, device=DEV).to(BF16)
    seqs = lram.pack([1, 1, 1])  # and a row of no sequence
    seqs = seqs._replace(start_q=seqs.start_q.clone())

    def step(cache, x):
        s = cache.extend(seqs)
        q = lram.paged_append(x[:, heads:heads + kv], x[:, heads + kv:], cache.keys[0], cache.table, s, q=x[:, :heads], rotary=plan)
        out = lram.paged_attention(q, cache.keys[0], cache.table, s, weigh=True)
        cache.evict(budget, 4)
        return out

    for c in (eager, captured):
        c.reserve([90, 90, 90])
        for t in c.keys[0][:2]:
            t.zero_()
        c.keys[0].position.zero_()
        c.keys[0].weight.zero_()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(2):
            step(captured, x)
    torch.cuda.current_stream().wait_stream(s)
    for _ in range(2):
        step(eager, x)
    eager.table.table.copy_(captured.table.table)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(captured, x)
    for lengths in ([1, 1, 1], [1, 0, 1], [2, 1, 1], [0, 0, 3], [1, 1, 1]) * 12:
        seqs.start_q.copy_(lram.pack(lengths).start_q)
        x.copy_(torch.randn(x.shape, generator=g, device=DEV))
        want = step(eager, x)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert torch.equal(captured.table.used, eager.table.used) and torch.equal(captured.table.seen, eager.table.seen)
        for a, b in zip(captured.keys[0], eager.keys[0]):
            assert _same(a, b)
    # once a step was captured, the host's calls go by the real lengths
    used = eager.table.used.tolist()
    captured.reserve([5, 5, 5])
    assert captured._used == used
    captured.trim()
    assert captured.free_pages() == 9 - sum(-(-n // 32) for n in used)
    assert captured.refresh() == eager.refresh() == used


def test_a_captured_eviction_is_no_cut_yet():
    """Only the eviction is captured: until it is replayed the host gives pages out by the lengths as they are."""
    cache = lram.PagedCache(1, 4, 1, 32, page=32, dtype=BF16, weigh=True)
    rows = torch.randn((60, 1, 32), generator=_gen(21), device=DEV).to(BF16)

    def append(n):
        lram.paged_append(rows[:n], rows[:n], cache.keys[0], cache.table, cache.extend(lram.pack([n])))

    append(60)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        lram.paged_evict(cache.keys[0], cache.table, 60)  # the first call of the kernels: nothing is over the budget
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.evict(30)
    append(10)
    assert len(lram.paged_read(cache.keys[0], cache.table, 0)[0]) == 70  # refuses where a page is missing
    graph.replay()
    append(5)
    assert cache.refresh() == [35]
    assert lram.paged_read(cache.keys[0], cache.table, 0)[2].flatten().tolist()[30:] == list(range(70, 75))


def test_two_streams_at_once():
    """Two readers of a cache and a writer of another, each on a stream of its own."""
    g = _gen(15)
    keys, table = _cache(g, [3000, 100], 2, 64, 64, BF16)
    other, others = _cache(g, [900, 2000], 2, 64, 64, BF16)
    q = torch.randn((2, 8, 64), generator=g, device=DEV).to(BF16)
    seqs = _plan([1, 1], max_k=3000)
    want = lram.paged_attention(q, keys, table, seqs)
    saved = other.weight.clone()
    lram.paged_attention(q, other, others, seqs, weigh=True)
    want_weight = other.weight.clone()
    other.weight.copy_(saved)
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for s in streams[:2]:
        with torch.cuda.stream(s):
            got.append([lram.paged_attention(q, keys, table, seqs) for _ in range(5)])
    with torch.cuda.stream(streams[2]):
        lram.paged_attention(q, other, others, seqs, weigh=True)
    for s in streams:
        torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(x, want) for r in got for x in r) and _same(other.weight, want_weight)


def test_refusals():
    g = _gen(16)
    keys, table = _cache(g, [10], 2, 64, 32, BF16)
    bare = keys._replace(weight=None)
    x = torch.zeros((1, 4, 64), dtype=BF16, device=DEV)
    k = x[:, :2]
    seqs = _plan([1])
    plan = lram.rotary_plan(64)

    def refused(what, call, *a, **kw):
        with pytest.raises(lram.LramError, match=what):
            call(*a, **kw)

    refused("multiple of the cache's", lram.paged_attention, x[:, :3], keys, table, seqs)
    refused("64 times", lram.paged_attention, x.new_zeros((1, 130, 64)), keys, table, seqs)
    refused("scale", lram.paged_attention, x, keys, table, seqs, scale=0.0)
    refused("no weights", lram.paged_attention, x, bare, table, seqs, weigh=True)
    refused("no weights", lram.paged_evict, bare, table, 4)
    refused("no weights", lram.paged_append, k, k, bare, table, seqs, weight=torch.zeros((1, 2), device=DEV))
    refused("device, type", lram.paged_attention, x.float(), keys, table, seqs)
    refused("device, type", lram.paged_append, k, k.float(), keys, table, seqs)
    refused("16 bytes", lram.paged_attention, x.new_zeros((1, 4, 72))[..., 4:68], keys, table, seqs)
    refused("of the cache", lram.paged_append, x[:, :3], x[:, :3], keys, table, seqs)
    refused("with k's rows", lram.paged_append, k, k, keys, table, seqs, q=x.new_zeros((2, 4, 64)), rotary=plan)
    refused("1 to head_dim / 2", lram.paged_append, k, k, keys, table, seqs, q=x, rotary=lram.rotary_plan(66))
    refused("start_q", lram.paged_attention, x, keys, table, _plan([1, 1]))
    refused("table", lram.paged_attention, x, keys, table._replace(table=table.table.long()), seqs)
    refused("recent", lram.paged_evict, keys, table, 4, 5)
    refused("at least 1", lram.paged_evict, keys, table, 0)
    refused("at least 1", lram.paged_shrink, table, 0)
    refused("v must", lram.paged_attention, x, keys._replace(v=keys.v[:1]), table, seqs)
    refused("workspace", lram.paged_evict, keys, table, 4, 0, torch.zeros(8, dtype=torch.uint8, device=DEV))
    rel = lram.RelativeBias(torch.zeros((4, 8), dtype=BF16, device=DEV), _ints([0] * 1857))
    refused("2 reach", lram.paged_attention, x, keys, table, seqs, rel=rel)
    refused("256 buckets", lram.paged_attention, x, keys, table, seqs,
            rel=lram.RelativeBias(torch.zeros((4, 257), dtype=BF16, device=DEV), _ints([0] * 3)))
