"""Host-side checks of rotary positions and the cache in pages: exports, argument checks of the C ABI (nothing is launched),
frequencies, and how the cache gives its pages out.  No GPU is needed."""
import ctypes
import math
import os
import re
import subprocess

import pytest
import torch

import paper_2107_03474_amd as lram
from paper_2107_03474_amd import paged, positions

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000      # never dereferenced: every call here ends in the host's checks
EINVAL, EDTYPE, EWORKSPACE = 1, 3, 4


@pytest.fixture(scope="module")
def lib():
    positions._library()
    return paged._library()


def test_every_declared_symbol_is_exported(lib):
    txt = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "lram_cache.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(lram_[a-z_0-9]+)\s*\(", txt))
    assert len(names) == 9
    out = subprocess.run(["nm", "-D", "--defined-only", lram.library_path()], capture_output=True, text=True, check=True).stdout
    assert names <= set(re.findall(r"\bT (lram_[a-z_0-9]+)", out))


def _rotation(pairs=32, interleaved=0, magnitude=1.0, turns=P):
    return positions._Rotary(pairs, interleaved, magnitude, turns)


def _rotate(lib, r=None, dt=1, rows=4, dim=64, at=P, q=P, q_row=512, q_head=64, heads=8, q_out=P, k=P, k_row=256, k_head=64, kv=4,
            k_out=P):
    return lib.lram_rotate(_rotation() if r is None else r, dt, 0, rows, dim, at, q, q_row, q_head, heads, q_out, k, k_row,
                           k_head, kv, k_out, None)


def test_rotate_refuses(lib):
    for bad in (dict(r=_rotation(0)), dict(r=_rotation(33)), dict(r=_rotation(interleaved=2)), dict(r=_rotation(magnitude=math.inf)),
                dict(r=_rotation(magnitude=math.nan)), dict(r=_rotation(turns=None)), dict(r=_rotation(turns=P + 4)), dict(rows=-1),
                dict(rows=(1 << 30) + 1), dict(dim=0), dict(dim=60), dict(dim=1032), dict(at=None), dict(at=P + 2), dict(q=None),
                dict(q=P + 8), dict(q_row=56), dict(q_row=516), dict(q_row=1 << 23), dict(q_head=-64), dict(q_head=4),
                dict(heads=0), dict(q_out=None), dict(q_out=P + 2), dict(k=None), dict(k_out=None), dict(k_row=4), dict(kv=-1)):
        assert _rotate(lib, **bad) == EINVAL, bad
    assert _rotate(lib, dt=2) == EDTYPE
    assert lib.lram_rotate(None, 1, 0, 4, 64, P, P, 512, 64, 8, P, None, 0, 0, 0, None, None) == EINVAL
    assert _rotate(lib, rows=0, q=None, k=None) == 0
    for bad in (dict(start=None), dict(start=P + 2), dict(batch=-1), dict(batch=1 << 25), dict(rows=-1), dict(out=None),
                dict(out=P + 1), dict(first=P + 2)):
        a = dict(dict(start=P, first=None, batch=3, rows=7, out=P), **bad)
        assert lib.lram_positions(a["start"], a["first"], a["batch"], a["rows"], a["out"], None) == EINVAL, bad
    assert lib.lram_positions(P, None, 3, 0, P, None) == 0


def _pool(**kw):
    a = paged._Paged(dtype=1, heads=8, kv_heads=4, head_dim=64, batch=2, page=64, pages=100, width=40, k=P, v=P, position=P,
                     weight=P, table=P, used=P, seen=P, start=P, rows=6, max_q=3, max_k=2000)
    for n, v in kw.items():
        setattr(a, n, v)
    return a


SHARED = [dict(kv_heads=0), dict(kv_heads=2048, heads=2048), dict(page=16), dict(page=48), dict(page=512), dict(batch=-1), dict(batch=1 << 21),
          dict(pages=-1), dict(pages=(1 << 24) + 1), dict(width=-1), dict(width=(1 << 24) + 1), dict(max_k=-1), dict(k=None), dict(v=None),
          dict(position=None), dict(k=P + 8), dict(v=P + 2), dict(position=P + 4), dict(weight=P + 4), dict(used=None), dict(seen=None),
          dict(table=None), dict(used=P + 2), dict(seen=P + 1), dict(table=P + 2)]
TYPES = [dict(dtype=2), dict(head_dim=48), dict(head_dim=256)]
NEW_ROWS = [dict(heads=0), dict(heads=6), dict(heads=65 * 4), dict(rows=-1), dict(rows=1 << 30), dict(max_q=-1), dict(start=None),
            dict(start=P + 2)]


def _append(lib, r=None, k=P, k_row=256, k_head=64, v=P, v_row=256, v_head=64, given=None, q=P, q_row=512, q_head=64, q_out=P, **kw):
    r = _rotation() if r is None else r or None
    return lib.lram_paged_append(_pool(**kw), r, k, k_row, k_head, v, v_row, v_head, given, q, q_row, q_head, q_out, None)


def test_append_and_extend_refuse(lib):
    for bad in SHARED + NEW_ROWS + [
            dict(k=P, weight=None, given=P), dict(given=P + 2), dict(k_row=60), dict(k_head=4), dict(v_row=1 << 23), dict(v_head=-64),
            dict(q=None), dict(q_out=None), dict(q=P + 2), dict(q_out=P + 8), dict(q_row=32), dict(q_head=4), dict(r=False),
            dict(r=_rotation(33)), dict(r=_rotation(turns=None))]:
        pool = {n: v for n, v in bad.items() if n in dict(paged._Paged._fields_)}
        rest = {n: v for n, v in bad.items() if n not in pool}
        assert _append(lib, **rest, **{n: v for n, v in pool.items() if n not in ("k", "v")}) == EINVAL if not {"k", "v"} & set(pool) \
            else lib.lram_paged_append(_pool(**pool), None, P, 256, 64, P, 256, 64, rest.get("given"), None, 0, 0, None, None) == EINVAL, bad
    for bad in (dict(k=None), dict(v=None), dict(k=P + 8), dict(v=P + 2)):
        assert _append(lib, **bad) == EINVAL, bad
    for bad in TYPES:
        assert _append(lib, **bad) == EDTYPE, bad
    assert lib.lram_paged_append(None, None, P, 256, 64, P, 256, 64, None, None, 0, 0, None, None) == EINVAL
    assert _append(lib, rows=0) == 0
    for bad in ((None, 2, P, P), (P, 2, None, P), (P, 2, P, None), (P, -1, P, P), (P + 2, 2, P, P), (P, 2, P + 1, P), (P, 1 << 21, P, P)):
        assert lib.lram_paged_extend(*bad, None) == EINVAL, bad
    assert lib.lram_paged_extend(None, 0, None, None, None) == 0


def _queries(**kw):
    a = paged._Queries(q=P, q_row=512, q_head=64, scale=0.125, weigh=0, wdtype=1)
    for n, v in kw.items():
        setattr(a, n, v)
    return a


BIAS = dict(rel_weight=P, rel_bucket=P, rel_buckets=32, rel_reach=128)


def test_attention_refuses(lib):
    n = ctypes.c_size_t(0)
    for bad in SHARED + NEW_ROWS:
        assert lib.lram_paged_attention(_pool(**bad), _queries(), P, P, 1 << 40, None) == EINVAL, bad
        assert lib.lram_paged_attention_workspace_bytes(_pool(**bad), _queries(), n) == EINVAL, bad
    for bad in TYPES:
        assert lib.lram_paged_attention(_pool(**bad), _queries(), P, P, 1 << 40, None) == EDTYPE, bad
    for bad in (dict(q=None), dict(q=P + 8), dict(q_row=60), dict(q_row=516), dict(q_head=4), dict(scale=0.0), dict(scale=math.nan),
                dict(scale=math.inf), dict(weigh=2), dict(BIAS, rel_bucket=None), dict(BIAS, rel_buckets=0), dict(BIAS, rel_buckets=257),
                dict(BIAS, rel_reach=-1), dict(BIAS, rel_reach=2000), dict(BIAS, rel_weight=P + 1), dict(BIAS, rel_bucket=P + 2)):
        assert lib.lram_paged_attention(_pool(), _queries(**bad), P, P, 1 << 40, None) == EINVAL, bad
    assert lib.lram_paged_attention(_pool(), _queries(**dict(BIAS, wdtype=5)), P, P, 1 << 40, None) == EDTYPE
    assert lib.lram_paged_attention(_pool(weight=None), _queries(weigh=1), P, P, 1 << 40, None) == EINVAL
    for out in (None, P + 8):
        assert lib.lram_paged_attention(_pool(), _queries(), out, P, 1 << 40, None) == EINVAL
    assert lib.lram_paged_attention(None, _queries(), P, P, 1 << 40, None) == EINVAL
    assert lib.lram_paged_attention(_pool(), None, P, P, 1 << 40, None) == EINVAL
    assert lib.lram_paged_attention_workspace_bytes(_pool(), _queries(), None) == EINVAL
    assert lib.lram_paged_attention_workspace_bytes(_pool(weight=P), _queries(weigh=1), n) == 0 and n.value >= 6 * 8 * 8
    for bad in ((None, 1 << 40), (P + 4, 1 << 40), (P, n.value - 1)):
        assert lib.lram_paged_attention(_pool(), _queries(weigh=1), P, *bad, None) == EWORKSPACE, bad
    assert lib.lram_paged_attention(_pool(rows=0), _queries(q=None), None, None, 0, None) == 0


@pytest.mark.parametrize("rows", [1, 1000, 100_000])
@pytest.mark.parametrize("max_q,max_k", [(0, 0), (1, 1 << 26), (1, 1 << 40), (1 << 40, 1 << 40)])
@pytest.mark.parametrize("batch", [1, 3000])
def test_workspaces_of_odd_expectations(lib, rows, max_q, max_k, batch):
    """What is expected never asks for more than twice the partial results of as many workgroups as fill the card, or of one
    piece a sequence."""
    n = ctypes.c_size_t(0)
    a = _pool(rows=rows, max_q=max_q, max_k=max_k, batch=batch, width=1 << 20)
    assert lib.lram_paged_attention_workspace_bytes(a, _queries(), n) == 0
    most = 2 * max(2048 * 64, rows * 8) * (64 + 2) * 4
    assert n.value <= most
    assert lib.lram_paged_attention_workspace_bytes(a, _queries(weigh=1), n) == 0
    assert n.value <= most + (256 << 20)  # and the scores of single tokens


def test_evict_refuses(lib):
    n = ctypes.c_size_t(0)
    for bad in SHARED:
        assert lib.lram_paged_evict(_pool(**bad), 100, 10, P, 1 << 40, None) == EINVAL, bad
    for bad in TYPES:
        assert lib.lram_paged_evict(_pool(**bad), 100, 10, P, 1 << 40, None) == EDTYPE, bad
    for budget, recent in ((0, 0), (-1, 0), (10, 11), (10, -1)):
        assert lib.lram_paged_evict(_pool(), budget, recent, P, 1 << 40, None) == EINVAL
    assert lib.lram_paged_evict(_pool(weight=None), 100, 10, P, 1 << 40, None) == EINVAL
    assert lib.lram_paged_evict_workspace_bytes(_pool(), 100, n) == 0 and n.value == 2 * 4 * (2 * 100 + 1) * 4
    for bad in ((None, 1 << 40), (P + 4, 1 << 40), (P, n.value - 1)):
        assert lib.lram_paged_evict(_pool(), 100, 10, *bad, None) == EWORKSPACE, bad
    assert lib.lram_paged_evict_workspace_bytes(_pool(), 2550, n) == 0 and n.value == 2 * 4 * (2 * 10 + 1) * 4  # 40 pages hold 2560
    assert lib.lram_paged_evict(_pool(), 2560, 10, None, 0, None) == 0  # nothing can be over the budget
    assert lib.lram_paged_evict(_pool(), 1 << 60, 10, None, 0, None) == 0
    assert lib.lram_paged_evict(_pool(batch=0), 100, 10, None, 0, None) == 0
    for bad in ((0, 3, P), (10, -1, P), (10, (1 << 20) + 1, P), (10, 3, None), (10, 3, P + 2)):
        assert lib.lram_paged_shrink(*bad, None) == EINVAL, bad
    assert lib.lram_paged_shrink(10, 0, None, None) == 0


def test_tensors_of_the_host_are_refused(lib):
    keys, table = lram.paged_keys(4, 2, 32, weigh=True, device="cpu"), lram.page_table(2, 2, device="cpu")
    seqs, rows = lram.pack([1, 1], device="cpu"), torch.zeros((2, 2, 32), dtype=torch.bfloat16)
    for call in (lambda: lram.paged_evict(keys, table, 1), lambda: lram.paged_shrink(table, 1), lambda: lram.paged_extend(table, seqs),
                 lambda: lram.paged_append(rows, rows, keys, table, seqs), lambda: lram.paged_attention(rows, keys, table, seqs),
                 lambda: lram.rotary_forward(rows, None, table.used, lram.rotary_plan(32, device="cpu"))):
        with pytest.raises(lram.LramError, match="GPU tensor"):
            call()


def test_frequencies():
    def of(**kw):
        p = lram.rotary_plan(16, device="cpu", **kw)
        return [(int(t) % (1 << 64)) / 2.0 ** 64 * 2 * math.pi for t in p.turns], p

    plain, p = of()
    assert p.magnitude == 1.0 and p.interleaved is False
    assert plain == pytest.approx([10000.0 ** (-i / 8) for i in range(8)], rel=1e-14)
    assert of(scaling="linear", factor=4.0)[0] == pytest.approx([f / 4 for f in plain], rel=1e-14)
    slow, _ = of(scaling="base", factor=4.0)
    assert slow[0] == pytest.approx(1.0) and slow[7] == pytest.approx(plain[7] / 4, rel=1e-12)
    parts, p = of(scaling="parts", factor=4.0, length=1000, low=2.0, high=50.0)
    assert p.magnitude == pytest.approx(0.1 * math.log(4.0) + 1)
    for f, g in zip(plain, parts):
        turns = 1000 * f / (2 * math.pi)
        s = min(max((turns - 2) / 48, 0), 1)
        assert g == pytest.approx(f * (s + (1 - s) / 4), rel=1e-12)
    fast = lram.rotary_plan(4, base=1e-3, device="cpu").turns.tolist()  # beyond a half turn a token: the fraction's upper bit
    assert (fast[1] % (1 << 64)) / 2.0 ** 64 == pytest.approx(math.sqrt(1000.0) / (2 * math.pi) % 1, rel=1e-12)
    for bad in (dict(dim=0), dict(dim=7), dict(dim=8, base=0.0), dict(dim=8, scaling="cubic"), dict(dim=8, scaling="linear", factor=0.0),
                dict(dim=8, scaling="parts", factor=2.0), dict(dim=2, scaling="base", factor=2.0),
                dict(dim=8, scaling="parts", factor=2.0, length=10, low=4.0, high=4.0)):
        with pytest.raises(lram.LramError):
            lram.rotary_plan(**bad, device="cpu")


def test_pages_are_given_out_and_back():
    c = lram.PagedCache(3, 10, 2, 32, page=32, capacity=100, dtype=torch.float32, device="cpu")
    assert c.capacity == 100 and c.table.table.shape == (3, 4) and c.free_pages() == 10
    c.reserve([33, 0, 1])
    assert c.free_pages() == 7 and (c.table.table >= 0).sum(1).tolist() == [2, 0, 1]
    c._used = [33, 0, 1]
    c.table.used.copy_(torch.tensor([33, 0, 1]))
    c.reserve([31, 32, 31])  # up to the pages' ends: one more page
    assert c.free_pages() == 6 and (c.table.table >= 0).sum(1).tolist() == [2, 1, 1]
    held = c.table.table[c.table.table >= 0].tolist()
    assert len(set(held)) == len(held)
    with pytest.raises(ValueError, match="capacity of 100"):
        c.reserve([68, 0, 0])
    c.reserve([67, 0, 0])
    assert c.free_pages() == 4
    with pytest.raises(ValueError, match="4 free pages, and 5 are needed"):
        c.reserve([0, 100, 64])
    assert c.free_pages() == 4 and (c.table.table >= 0).sum(1).tolist() == [4, 1, 1]  # nothing was given out
    c.trim()
    assert c.free_pages() == 7 and (c.table.table >= 0).sum(1).tolist() == [2, 0, 1]
    c._used = [100, 100, 100]  # bounds that are too high: the lengths are read back
    c.reserve([67, 0, 0])
    assert c._used == [33, 0, 1]
    c.release([0, 2])
    assert c.free_pages() == 10 and (c.table.table < 0).all() and c.table.used.tolist() == [0, 0, 0]
    c.reserve([32, 0, 70])
    c.table.used.copy_(torch.tensor([33, 0, 70]))  # a replayed step went on past what was reserved
    c._captured = True
    for call in (c.refresh, c.trim, lambda: c.reserve([0, 0, 0])):
        with pytest.raises(lram.LramError, match="sequence 0 has counted 33 keys, and 32 were reserved"):
            call()
    c.release([0])
    c.reserve([0, 0, 30])
    assert c.free_pages() == 6 and c.refresh() == [0, 0, 70]
    c.table.used[2] = 101
    with pytest.raises(lram.LramError, match="101 keys, and 100 were"):
        c.refresh()
    c.release([0, 2])
    for bad in ([1, 2], [1, 2, -3]):
        with pytest.raises(ValueError, match="lengths"):
            c.reserve(bad)
    with pytest.raises(ValueError, match="3 sequences"):
        c.release([3])
    with pytest.raises(ValueError, match="3 sequences"):
        c.extend(lram.pack([1, 1], device="cpu"))
    for bad in (dict(page=16), dict(head_dim=48), dict(kv_heads=0), dict(pages=1 << 30), dict(dtype=torch.float16)):
        with pytest.raises(lram.LramError):
            lram.paged_keys(**dict(dict(pages=2, kv_heads=1, head_dim=32, device="cpu"), **bad))
