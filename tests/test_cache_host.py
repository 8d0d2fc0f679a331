"""The key-value cache's bookkeeping, on CPU tensors."""
import pytest
import torch

import paper_2107_03474_amd as lram
from paper_2107_03474_amd.memory_block import KeyValueCache


def _cache(batch, capacity):
    c = KeyValueCache(batch, capacity, 1, 2, torch.float32, device="cpu")
    c.k.fill_(-1.0)
    c.v.fill_(-2.0)
    return c


def _rows(n, first=1):
    k = torch.arange(first, first + n).float()[:, None, None].expand(n, 1, 2).contiguous()
    return k, -10 * k


def _pack(n, front=0):
    p = lram.pack(n, device="cpu")
    return p._replace(start_q=p.start_q + front)


def _holds(cache, want):
    """want: the first numbers of each sequence's keys; all else untouched."""
    full = torch.full((cache.batch, cache.capacity), -1.0)
    for b, rows in enumerate(want):
        full[b, :len(rows)] = torch.tensor(rows)
    assert torch.equal(cache.k[:, 0, 0].view(cache.batch, cache.capacity), full)
    assert torch.equal(cache.v[:, 0, 1].view(cache.batch, cache.capacity), torch.where(full < 0, -2.0, -10 * full))


def test_rows_join_their_sequences():
    c = _cache(3, 5)
    seqs = c.append(*_rows(5), _pack([2, 0, 3]))
    _holds(c, [[1, 2], [], [3, 4, 5]])
    assert c.used.tolist() == seqs.used_k.tolist() == [2, 0, 3] and seqs.start_k.tolist() == [0, 5, 10, 15]
    assert c.k.shape == (15, 1, 2) and c.v.shape == (15, 1, 2)
    c.append(*_rows(4, 6), _pack([1, 2, 1]))
    _holds(c, [[1, 2, 6], [7, 8], [3, 4, 5, 9]])
    assert c.used.tolist() == [3, 2, 4]


@pytest.mark.parametrize("front,behind", [(0, 3), (2, 0), (1, 4)])
def test_rows_of_no_sequence_are_left_out(front, behind):
    c = _cache(2, 4)
    for step in range(2):
        n = front + 3 + behind
        c.append(*_rows(n, 1 + 10 * step), _pack([1, 2], front))
    _holds(c, [[1 + front, 11 + front], [2 + front, 3 + front, 12 + front, 13 + front]])
    assert c.used.tolist() == [2, 4]


def test_a_sequence_that_outgrows_the_cache_is_refused_and_changes_nothing():
    c = _cache(2, 4)
    c.append(*_rows(5), _pack([3, 2]))
    for n in ([2, 0], [0, 3], [4, 4]):
        with pytest.raises(ValueError, match="capacity"):
            c.append(*_rows(sum(n), 6), _pack(n))
        _holds(c, [[1, 2, 3], [4, 5]])
        assert c.used.tolist() == [3, 2]
    c.append(*_rows(3, 6), _pack([1, 2]))
    _holds(c, [[1, 2, 3, 6], [4, 5, 7, 8]])


def test_long_texts_one_after_the_other_are_not_refused():
    """Each within the capacity, though the longest of the calls add up to more."""
    c = _cache(3, 4)
    for b in range(3):
        n = [4 if i == b else 0 for i in range(3)]
        c.append(*_rows(4, 1 + 4 * b), _pack(n))
    _holds(c, [[1, 2, 3, 4], [5, 6, 7, 8], [9, 10, 11, 12]])


def test_what_passes_the_capacity_unseen_reaches_no_other_sequence():
    """Lengths that the plan's max_q understates, as when a captured call is replayed over others: the rows past the capacity
    are left out."""
    c = _cache(2, 4)
    c.append(*_rows(7), _pack([6, 1])._replace(max_q=1))
    _holds(c, [[1, 2, 3, 4], [7]])
    assert c.used.tolist() == [4, 1]


def test_refuses():
    c = _cache(2, 4)
    k, v = _rows(3)
    for bad in ((k, v, _pack([3])), (k, v, _pack([1, 1, 1])), (k[:2], v, _pack([1, 2])), (k.expand(3, 2, 2), v, _pack([1, 2])),
                (k, v[..., :1], _pack([1, 2])), (k[:2], v[:2], _pack([1, 2])._replace(start_q=torch.zeros(1, dtype=torch.int32)))):
        with pytest.raises(ValueError):
            c.append(*bad)
    for bad in ((-1, 4), (2, -1), (1 << 16, 1 << 15)):
        with pytest.raises(ValueError):
            KeyValueCache(*bad, 1, 2, device="meta")
