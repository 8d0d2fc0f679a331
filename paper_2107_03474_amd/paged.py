"""A key-value cache in pages for serving the layer around the lattice memory: new rows into it (with their rotation), attention
of new tokens over it, and eviction from it by accumulated attention weight.

As in the package's other calls, this module only marshals torch tensors and the current HIP stream into the C ABI
(``include/lram_cache.h``, which says where a key lies in its page); there is no fallback.  Sums, statistics and weights are fp32.
In bf16 attention's softmax weights enter the product with the values with 16 bits where a call expects at most 16 new rows times
heads / kv_heads of a sequence, otherwise rounded to bf16.
"""
from __future__ import annotations

import ctypes
import math
from typing import List, NamedTuple, Optional, Sequence, Tuple

import torch
from torch.autograd import forward_ad

from . import F32, LramError
from . import load as _load_library
from .layer import HEAD_DIMS, Packed, RelativeBias, _check, _heads, _ptr, _scratch, _type
from .positions import Rotary, _launch, _refusal, _Rotary, _rotary

__all__ = ["PagedKeys", "PageTable", "paged_keys", "page_table", "paged_extend", "paged_append", "paged_attention",
           "paged_evict", "paged_shrink", "paged_read", "PagedCache"]

_P, _I64, _I32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32
PAGE_SIZES = (32, 64, 128, 256)


class _Paged(ctypes.Structure):
    """lram_paged"""
    _fields_ = ([(n, _I32) for n in ("dtype", "heads", "kv_heads", "head_dim", "batch", "page")] +
                [(n, _I64) for n in ("pages", "width")] +
                [(n, _P) for n in ("k", "v", "position", "weight", "table", "used", "seen", "start")] +
                [(n, _I64) for n in ("rows", "max_q", "max_k")])


class _Queries(ctypes.Structure):
    """lram_paged_queries"""
    _fields_ = ([("q", _P), ("q_row", _I64), ("q_head", _I64), ("scale", ctypes.c_float)] +
                [(n, _I32) for n in ("weigh", "wdtype", "rel_buckets", "rel_reach")] + [("rel_weight", _P), ("rel_bucket", _P)])


_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = _load_library()
        A, Q, R = ctypes.POINTER(_Paged), ctypes.POINTER(_Queries), ctypes.POINTER(_Rotary)
        SZ, SZP = ctypes.c_size_t, ctypes.POINTER(ctypes.c_size_t)
        lib.lram_paged_extend.argtypes = [_P, _I32, _P, _P, _P]
        lib.lram_paged_append.argtypes = [A, R, _P, _I64, _I64, _P, _I64, _I64, _P, _P, _I64, _I64, _P, _P]
        lib.lram_paged_attention_workspace_bytes.argtypes = [A, Q, SZP]
        lib.lram_paged_attention.argtypes = [A, Q, _P, _P, SZ, _P]
        lib.lram_paged_evict_workspace_bytes.argtypes = [A, _I64, SZP]
        lib.lram_paged_evict.argtypes = [A, _I64, _I64, _P, SZ, _P]
        lib.lram_paged_shrink.argtypes = [_I64, _I32, _P, _P]
        _lib = lib
    return _lib


class PagedKeys(NamedTuple):
    """The pages of one layer.  With e = 16 bytes of elements (8 in bf16, 4 in fp32) and keys t = 0 ... page - 1 of a page:
    k [pages, kv_heads, page / 16, head_dim / e, 16, e] holds key t, dimension d at [t / 16, d / e, t % 16, d % e];
    v [pages, kv_heads, page / 4e, head_dim / 16, 4, 16, e] at [t / 4e, d / 16, t % 16 / 4, d % 16, t % 4e / 16 * 4 + t % 4];
    position and weight [pages, kv_heads, page] (int32; fp32, None where keys gather no weight) its place in its text and the
    attention weight that it has gathered."""
    k: torch.Tensor
    v: torch.Tensor
    position: torch.Tensor
    weight: Optional[torch.Tensor] = None


class PageTable(NamedTuple):
    """Which pages hold which sequence, for all layers (int32 device tensors): table [batch, width] names the pages of each in
    their order (-1: none yet), used [batch] counts its keys, seen [batch] the tokens that it has had.  No page belongs to two
    sequences."""
    table: torch.Tensor
    used: torch.Tensor
    seen: torch.Tensor


def paged_keys(pages: int, kv_heads: int, head_dim: int, page: int = 64, dtype=torch.bfloat16, weigh: bool = False,
               device="cuda") -> PagedKeys:
    """Pages for one layer, not filled; weigh: with weights."""
    if page not in PAGE_SIZES or head_dim not in HEAD_DIMS or dtype not in (torch.float32, torch.bfloat16):
        raise LramError("pages hold 32, 64, 128 or 256 keys of head_dim 32, 64 or 128 in float32 or bfloat16")
    if pages < 0 or pages * page > 1 << 30 or not 1 <= kv_heads <= 1024:
        raise LramError("pages hold 2^30 keys at most, of 1 to 1024 heads")
    e = 16 // torch.empty((), dtype=dtype).element_size()
    new = dict(dtype=dtype, device=device)
    return PagedKeys(torch.empty((pages, kv_heads, page // 16, head_dim // e, 16, e), **new),
                     torch.empty((pages, kv_heads, page // (4 * e), head_dim // 16, 4, 16, e), **new),
                     torch.empty((pages, kv_heads, page), dtype=torch.int32, device=device),
                     torch.empty((pages, kv_heads, page), dtype=torch.float32, device=device) if weigh else None)


def page_table(batch: int, width: int, device="cuda") -> PageTable:
    """A table of empty sequences, of at most ``width`` pages each."""
    i32 = dict(dtype=torch.int32, device=device)
    return PageTable(torch.full((batch, width), -1, **i32), torch.zeros(batch, **i32), torch.zeros(batch, **i32))


def _describe(keys: PagedKeys, table: PageTable, heads: int = 0, rows: int = 0, seqs: Optional[Packed] = None) -> _Paged:
    k, v, position, weight = keys
    where, used, seen = table
    of_k, of_position, of_table, of_used = k.shape, position.shape, where.shape, used.shape
    if len(of_k) != 6 or len(of_position) != 3:
        raise LramError("keys must be PagedKeys: k [pages, kv_heads, page / 16, head_dim / e, 16, e]")
    if not k.is_cuda:
        raise LramError("keys must be GPU tensors")
    dt, i32, on = k.dtype, torch.int32, k.get_device()
    code, e = _type(k, "k"), 8 if dt is torch.bfloat16 else 4
    pages, kv, page = of_position
    dim = of_k[3] * e
    if page not in PAGE_SIZES or dim not in HEAD_DIMS:
        raise LramError("pages hold 32, 64, 128 or 256 keys of head_dim 32, 64 or 128")
    if len(of_table) != 2 or len(of_used) != 1:
        raise LramError("table must be [batch, width], used and seen [batch]")
    batch, width = of_used[0], of_table[1]
    as_k, as_v = (pages, kv, page // 16, of_k[3], 16, e), (pages, kv, page // (4 * e), dim // 16, 4, 16, e)
    # one test for what is right, since small calls are bound by the host: a call for each tensor takes 1.5 us more
    if not (of_k == as_k and k.is_contiguous() and
            v.shape == as_v and v.dtype is dt and v.get_device() == on and v.is_contiguous() and
            position.dtype is i32 and position.get_device() == on and position.is_contiguous() and
            (weight is None or weight.shape == of_position and weight.dtype is torch.float32 and weight.get_device() == on and
             weight.is_contiguous()) and
            of_table[0] == batch and where.dtype is i32 and where.get_device() == on and where.is_contiguous() and
            used.dtype is i32 and used.get_device() == on and used.is_contiguous() and
            seen.shape == of_used and seen.dtype is i32 and seen.get_device() == on and seen.is_contiguous()):
        _ptr(k, "k", dt, as_k, k)  # one of these says what is wrong
        _ptr(v, "v", dt, as_v, k)
        _ptr(position, "position", i32, of_position, k)
        if weight is not None:
            _ptr(weight, "weight", torch.float32, of_position, k)
        _ptr(where, "table", i32, (batch, width), k)
        _ptr(used, "used", i32, (batch,), k)
        _ptr(seen, "seen", i32, (batch,), k)
    start = max_q = max_k = 0
    if seqs is not None:
        start, max_q, max_k = _ptr(seqs.start_q, "start_q", i32, (batch + 1,), k), seqs.max_q, seqs.max_k
    return _Paged(code, heads or kv, kv, dim, batch, page, pages, width, k.data_ptr(), v.data_ptr(), position.data_ptr(),
                  None if weight is None else weight.data_ptr(), where.data_ptr(), used.data_ptr(), seen.data_ptr(), start or None,
                  rows, max_q, max_k)


def _differentiated(*inputs: Optional[torch.Tensor]) -> bool:
    """Whether a derivative of these inputs is asked for, backward or by a tangent (no_grad leaves tangents as they are)."""
    inputs = [t for t in inputs if t is not None]
    return (torch.is_grad_enabled() and any(t.requires_grad for t in inputs) or
            forward_ad._current_level >= 0 and any(forward_ad.unpack_dual(t).tangent is not None for t in inputs))


def _like_keys(t: torch.Tensor, name: str, keys: PagedKeys, dim: int):
    """(address, row stride, head stride) of new rows that go with the cache."""
    k, shape = keys.k, t.shape
    if len(shape) == 3 and shape[2] == dim and t.dtype is k.dtype and t.get_device() == k.get_device() and t.is_cuda:
        row, head, one = t.stride()
        if one == 1:  # a dimension of size 1 has no stride to speak of
            return t.data_ptr(), row if shape[0] > 1 else shape[1] * dim, head if shape[1] > 1 else dim
    place = _heads(t, name, t)  # says what is wrong
    if t.dtype is not k.dtype or t.device != k.device or shape[2] != dim:
        raise LramError("%s must have the cache's device, type and head_dim" % name)
    return place


def _refused(rc: int, a: _Paged, dtype, places, rotary: Optional[Rotary] = None, rel: Optional[RelativeBias] = None,
             scale: float = 1.0):
    """Raises what the library refused, in the caller's terms where they can be told."""
    why = None
    if rc in (1, 3):
        per = 8 if dtype is torch.bfloat16 else 4
        if a.kv_heads > 1024 or a.heads % a.kv_heads or a.heads > 64 * a.kv_heads:
            why = "q's heads must be a multiple of the cache's, at most 64 times as many"
        elif not 0 < scale < math.inf:
            why = "scale must be positive and finite"
        elif any(p % 16 or row % per or head % per or head < 0 or not a.head_dim <= row <= 1 << 22 for p, row, head in places):
            why = ("new rows must start on 16 bytes, with strides of whole 16 bytes and rows at least head_dim and at most 2^22 "
                   "elements apart")
        elif rotary is not None:
            why = _refusal(dtype, a.head_dim, rotary, [])
        elif rel is not None and not 1 <= rel.weight.shape[1] <= 256:
            why = "a relative bias has 1 to 256 buckets"
        elif rel is not None and a.heads // a.kv_heads * (rel.bucket.shape[0] - 1 + 193) > 4096:
            why = "heads / kv_heads (2 reach + 193) must be at most 4096 with a relative bias"
    if why:
        raise LramError(why)
    _check(rc)


def paged_extend(table: PageTable, seqs: Packed) -> None:
    """used and seen grow by the sequences' new rows (packed by seqs.start_q): once a step, before its rows are appended to
    every layer's pages."""
    start, i32 = seqs.start_q, torch.int32
    batch = start.numel() - 1
    rc = _launch(start.device, _library().lram_paged_extend, _ptr(start, "start_q", i32, (batch + 1,), start), batch,
                 _ptr(table.used, "used", i32, (batch,), start), _ptr(table.seen, "seen", i32, (batch,), start))
    if rc:
        _check(rc)


def paged_append(k: torch.Tensor, v: torch.Tensor, keys: PagedKeys, table: PageTable, seqs: Packed,
                 q: Optional[torch.Tensor] = None, rotary: Optional[Rotary] = None, weight: Optional[torch.Tensor] = None
                 ) -> Optional[torch.Tensor]:
    """The new rows k and v [rows, kv_heads, head_dim] (packed by seqs.start_q; rows of no sequence are left out) into their
    pages: the last places of those that ``paged_extend`` has counted.  Keys are rotated by ``rotary`` at their positions; with
    weight [rows, kv_heads] fp32 they begin with these weights, not with 0.  Returns q [rows, heads, head_dim] rotated (q
    itself without a rotation, None without q).  Only start_q and max_q of seqs are used."""
    lib = _library()
    if _differentiated(k, v, q):
        raise LramError("a cache has no gradients: append to it under torch.no_grad()")
    rows = k.shape[0]
    a = _describe(keys, table, q.shape[1] if q is not None and q.dim() == 3 else 0, rows, seqs)
    dim = a.head_dim
    pk, pv = _like_keys(k, "k", keys, dim), _like_keys(v, "v", keys, dim)
    if k.shape != v.shape or k.shape[1] != a.kv_heads:
        raise LramError("k and v must be [rows, kv_heads, head_dim] of the cache")
    places, pq, out = [pk, pv], (None, 0, 0), q
    r = None if rotary is None else _rotary(rotary, k)
    if q is not None:
        pq = _like_keys(q, "q", keys, dim)
        if q.shape[0] != rows or not q.shape[1]:
            raise LramError("q must be [rows, heads, head_dim] with k's rows")
        places.append(pq)
        if rotary is None:
            pq = (None, 0, 0)
        else:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
    given = None
    if weight is not None:
        if keys.weight is None:
            raise LramError("the cache gathers no weights")
        given = _ptr(weight, "weight", torch.float32, (rows, a.kv_heads), k)
    rc = _launch(k.device, lib.lram_paged_append, a, r, *pk, *pv, given, *pq, out.data_ptr() if pq[0] is not None else None)
    if rc:
        _refused(rc, a, k.dtype, places, rotary)
    return out


def paged_attention(q: torch.Tensor, keys: PagedKeys, table: PageTable, seqs: Packed, scale: Optional[float] = None,
                    rel: Optional[RelativeBias] = None, weigh: bool = False, workspace: Optional[torch.Tensor] = None
                    ) -> torch.Tensor:
    """softmax(scale q k^T + bias) v of each sequence's new rows (q [rows, heads, head_dim], packed by seqs.start_q) over the
    keys in its pages whose positions are not past theirs; the bias is that of the distance between positions, the scale
    1 / sqrt(head_dim) by default.  weigh: the weights that each key is given, summed over queries and the heads that share
    it, are added to keys.weight.  Of seqs start_q, max_q and max_k are used; the work is divided by the longest, so that single
    tokens over long texts are served faster in a call without prompts."""
    lib = _library()
    if _differentiated(q, None if rel is None else rel.weight):
        raise LramError("attention over a cache has no gradients: call it under torch.no_grad()")
    if q.dim() != 3:
        raise LramError("q must be [rows, heads, head_dim]")
    rows, heads, dim = q.shape
    a = _describe(keys, table, heads, rows, seqs)
    place = _like_keys(q, "q", keys, a.head_dim)
    if not heads:
        raise LramError("q must have heads")
    if weigh and keys.weight is None:
        raise LramError("the cache gathers no weights")
    s = 1.0 / math.sqrt(dim) if scale is None else scale
    x = _Queries(*place, s, 1 if weigh else 0)
    if rel is not None:
        w, bucket = rel
        if w.dim() != 2 or bucket.dim() != 1 or bucket.numel() % 2 != 1:
            raise LramError("a relative bias has weight [heads, buckets] and bucket [2 reach + 1]")
        if w.dtype is not q.dtype and w.dtype is not torch.float32:
            raise LramError("the relative bias's weight must be float32 or of q's type")
        x.rel_weight = _ptr(w, "rel.weight", w.dtype, (heads, w.shape[1]), q)
        x.rel_bucket = _ptr(bucket, "rel.bucket", torch.int32, (bucket.shape[0],), q)
        x.wdtype, x.rel_buckets, x.rel_reach = _type(w, "rel.weight"), w.shape[1], bucket.shape[0] // 2
    out = torch.empty_like(q, memory_format=torch.contiguous_format)
    n = ctypes.c_size_t(0)
    rc = 0
    if workspace is None:
        rc = lib.lram_paged_attention_workspace_bytes(a, x, n)
    if not rc:
        ws, ws_bytes, keep = _scratch(n.value, workspace, q)
        rc = _launch(q.device, lib.lram_paged_attention, a, x, out.data_ptr(), ws, ws_bytes)
        del keep
    if rc:
        _refused(rc, a, q.dtype, [place], rel=rel, scale=s)
    return out


def paged_evict(keys: PagedKeys, table: PageTable, budget: int, recent: int = 0, workspace: Optional[torch.Tensor] = None
                ) -> None:
    """Cuts every sequence that uses more than ``budget`` keys down to it, each key head by itself: its keys of the ``recent``
    newest positions stay, and of the others those that have gathered the largest weights (at equal weights the lowest
    position; NaN is less than any).  Keys that stay past slot ``budget`` move into the slots that are left below it.  The
    lengths stay as they are, for the other layers: ``paged_shrink`` follows the last of them, before anything else is done
    with the cache."""
    lib = _library()
    if keys.weight is None:
        raise LramError("the cache gathers no weights")
    if not 0 <= recent <= budget or not 1 <= budget < 1 << 62:
        raise LramError("a budget is at least 1, and 0 <= recent <= budget")
    a = _describe(keys, table)
    n = ctypes.c_size_t(0)
    if workspace is None:
        _check(lib.lram_paged_evict_workspace_bytes(a, budget, n))
    ws, ws_bytes, keep = _scratch(n.value, workspace, keys.k)
    rc = _launch(keys.k.device, lib.lram_paged_evict, a, budget, recent, ws, ws_bytes)
    del keep
    if rc:
        _check(rc)


def paged_shrink(table: PageTable, budget: int) -> None:
    """used = min(used, budget): once every layer's pages are cut down to the budget."""
    if not 1 <= budget < 1 << 62:
        raise LramError("a budget is at least 1")
    used = table.used
    batch = used.numel()
    rc = _launch(used.device, _library().lram_paged_shrink, budget, batch, _ptr(used, "used", torch.int32, (batch,), used))
    if rc:
        _check(rc)


def paged_read(keys: PagedKeys, table: PageTable, b: int) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
    """(k, v [used, kv_heads, head_dim], position, weight [used, kv_heads]) of sequence b as plain tensors (copies; waits for the
    device)."""
    _, kv, page = keys.position.shape
    n = min(max(int(table.used[b]), 0), table.table.shape[1] * page)
    where = table.table[b, :(n + page - 1) // page].long()
    if n and not bool(((where >= 0) & (where < keys.k.shape[0])).all()):
        raise LramError("a page that sequence %d uses is missing" % b)
    k = keys.k[where].permute(0, 2, 4, 1, 3, 5).reshape(-1, kv, keys.k.shape[3] * keys.k.shape[5])
    v = keys.v[where].unflatten(-1, (-1, 4)).permute(0, 2, 6, 4, 7, 1, 3, 5).reshape(-1, kv, keys.v.shape[3] * 16)
    at, w = (None if t is None else t[where].transpose(1, 2).reshape(-1, kv)[:n] for t in (keys.position, keys.weight))
    return k[:n], v[:n], at, w


class PagedCache:
    """Keys and values of up to ``batch`` sequences and ``layers`` layers in pages that a pool of ``pages`` gives out as they are
    needed; a sequence holds ``capacity`` keys at most (the whole pool by default).  A step is

        seqs = cache.extend(seqs)        # pages for the new rows, and their places
        for each layer i: paged_append(k, v, cache.keys[i], cache.table, seqs, ...); paged_attention(q, cache.keys[i], ...)
        cache.evict(budget, recent)      # where the cache has weights and a budget

    The lengths are on the device.  The host keeps bounds of them, by which pages are given out.  A captured step takes only
    what was reserved before; once there was one, the host's calls read the lengths back first (``refresh``)."""

    def __init__(self, batch: int, pages: int, kv_heads: int, head_dim: int, page: int = 64, capacity: int = 0, layers: int = 1,
                 dtype=torch.bfloat16, weigh: bool = False, device="cuda"):
        if batch < 0 or pages < 0 or capacity < 0 or layers < 1:
            raise ValueError("a cache has sequences, pages, a capacity and at least one layer")
        width = min(-(-capacity // page), pages) if capacity else pages
        self.batch, self.page, self.capacity = batch, page, min(capacity, width * page) if capacity else width * page
        self.keys = [paged_keys(pages, kv_heads, head_dim, page, dtype, weigh, device) for _ in range(layers)]
        self.table = page_table(batch, width, device)
        self._host = torch.full((batch, width), -1, dtype=torch.int32)
        self._free = list(range(pages - 1, -1, -1))
        self._own: List[List[int]] = [[] for _ in range(batch)]
        self._used = [0] * batch  # no sequence uses more keys
        self._captured = False    # a step was captured, so that its replays may have changed the lengths

    def free_pages(self) -> int:
        return len(self._free)

    def refresh(self) -> List[int]:
        """The sequences' lengths, read back (waits for the device).  Refused where captured steps have counted rows past what
        was reserved, which are not in the cache: ``release`` ends such sequences."""
        used = self.table.used.tolist()
        for b, (n, own) in enumerate(zip(used, self._own)):
            if n > min(self.capacity, len(own) * self.page):
                raise LramError("sequence %d has counted %d keys, and %d were reserved" %
                                (b, n, min(self.capacity, len(own) * self.page)))
        self._used = used
        return list(used)

    def _missing(self, lengths) -> Tuple[Optional[str], List[int]]:
        more = [max(0, -(-(u + n) // self.page) - len(own)) for u, n, own in zip(self._used, lengths, self._own)]
        if any(n and u + n > self.capacity for u, n in zip(self._used, lengths)):
            return "a sequence has more rows than the cache's capacity of %d" % self.capacity, more
        if sum(more) > len(self._free):
            return "the cache has %d free pages, and %d are needed" % (len(self._free), sum(more)), more
        return None, more

    def reserve(self, lengths: Sequence[int]) -> None:
        """Pages for so many more rows of each sequence."""
        lengths = [int(n) for n in lengths]
        if len(lengths) != self.batch or any(n < 0 for n in lengths):
            raise ValueError("lengths must be those of the cache's %d sequences" % self.batch)
        if self._captured:
            self.refresh()
        why, more = self._missing(lengths)
        if why:  # the bounds may be too high
            self.refresh()
            why, more = self._missing(lengths)
            if why:
                raise ValueError(why)
        if any(more):
            for b, n in enumerate(more):
                for _ in range(n):
                    page = self._free.pop()
                    self._host[b, len(self._own[b])] = page
                    self._own[b].append(page)
            self.table.table.copy_(self._host)

    def extend(self, seqs: Packed, lengths: Optional[Sequence[int]] = None) -> Packed:
        """Counts the new rows that seqs packs (start_q), with pages for them; the plan of the step's appends and attention.
        lengths: the numbers of them, where the host knows them (else every sequence is taken to have max_q, which must then
        be no less)."""
        if seqs.start_q.numel() != self.batch + 1:
            raise ValueError("the plan must be of the cache's %d sequences" % self.batch)
        if torch.cuda.is_current_stream_capturing():
            self._captured = True
            paged_extend(self.table, seqs)
            return seqs._replace(max_k=min(self.capacity, max(map(len, self._own), default=0) * self.page))
        lengths = [seqs.max_q] * self.batch if lengths is None else lengths
        self.reserve(lengths)
        paged_extend(self.table, seqs)
        self._used = [u + int(n) for u, n in zip(self._used, lengths)]
        return seqs._replace(max_k=max(self._used, default=0))

    def evict(self, budget: int, recent: int = 0) -> None:
        """``paged_evict`` in every layer; the pages past the budget stay the sequences' own (``trim`` gives them back)."""
        for keys in self.keys:
            paged_evict(keys, self.table, budget, recent)
        paged_shrink(self.table, budget)
        if torch.cuda.is_current_stream_capturing():  # nothing is cut yet
            self._captured = True
        else:
            self._used = [min(u, budget) for u in self._used]

    def _give_back(self, keep: Sequence[int]) -> None:
        for b, n in enumerate(keep):
            while len(self._own[b]) > n:
                self._free.append(self._own[b].pop())
                self._host[b, len(self._own[b])] = -1
        self.table.table.copy_(self._host)

    def trim(self) -> None:
        """Pages that hold no key go back to the pool (waits for the device)."""
        self.refresh()
        self._give_back([-(-u // self.page) for u in self._used])

    def release(self, sequences: Sequence[int]) -> None:
        """These sequences end: their pages go back to the pool, and others may begin in their places."""
        gone = {int(b) for b in sequences}
        if any(not 0 <= b < self.batch for b in gone):
            raise ValueError("the cache has %d sequences" % self.batch)
        if not gone:
            return
        at = torch.tensor(sorted(gone)).to(self.table.used.device)
        self.table.used.index_fill_(0, at, 0)
        self.table.seen.index_fill_(0, at, 0)
        self._used = [0 if b in gone else u for b, u in enumerate(self._used)]
        self._give_back([0 if b in gone else len(own) for b, own in enumerate(self._own)])
