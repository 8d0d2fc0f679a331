"""A transformer layer whose feed-forward part is the lattice memory (Sec. 3.1, 3.2: the memory subnetwork replaces the
dense feed-forward part of one layer of a BERT-style model).

    a = attention(x);  x = norm(x + a);  x = norm(x + memory(x))

over packed sequences of different lengths, in both directions or causal, with a learned relative position bias or rotary
positions.  The attention, its bias, the rotation, the caches' pages, the norms with their residual adds and the lookup run in
liblram's kernels; the projections are library GEMMs.
"""
from __future__ import annotations

import math
from typing import Optional, Sequence, Union

import torch

from .layer import (HEAD_DIMS, Packed, RelativeBias, attention, attention_forward, bias_refusal, layer_norm,
                    relative_buckets)
from .memory_layer import MemorySubnetwork
from .paged import PagedCache, paged_append, paged_attention
from .positions import Rotary, packed_positions, rotary as rotate, rotary_forward


class KeyValueCache:
    """Keys and values of ``batch`` sequences, ``capacity`` rows each; ``used`` [batch] int32 counts the rows in use."""

    def __init__(self, batch: int, capacity: int, kv_heads: int, head_dim: int, dtype=torch.bfloat16, device="cuda"):
        if batch < 0 or capacity < 0 or batch * capacity > 1 << 30:
            raise ValueError("a cache holds batch * capacity rows, 2^30 at most")
        self.batch, self.capacity = batch, capacity
        # one row more, which takes what belongs to no sequence
        self._k = torch.empty((batch * capacity + 1, kv_heads, head_dim), dtype=dtype, device=device)
        self._v = torch.empty_like(self._k)
        self.k, self.v = self._k[:-1], self._v[:-1]
        self.used = torch.zeros(batch, dtype=torch.int32, device=device)
        self.start = torch.arange(batch + 1, dtype=torch.int32, device=device) * capacity
        # of the rows before the first sequence, of each sequence and past the last one: the end of its place in the cache
        self._end = torch.zeros(batch + 2, dtype=torch.int32, device=device)
        self._end[1:-1] = self.start[1:]
        self._base = torch.zeros_like(self._end)
        self._longest = 0  # no sequence has more rows, as far as the plans' max_q can be trusted

    def append(self, k: torch.Tensor, v: torch.Tensor, seqs: Packed) -> Packed:
        """Adds the rows of k and v (packed by seqs.start_q; rows of no sequence are left out) to their sequences; the plan of
        attention over the cache.  A sequence that would outgrow the capacity is refused, and nothing is added; the lengths
        are on the device, so that this is found by seqs.max_q, and where that is too low, or in a captured call, the rows
        past the capacity are left out."""
        if k.shape != v.shape or k.shape[1:] != self.k.shape[1:]:
            raise ValueError("k and v must be [rows, kv_heads, head_dim] of the cache")
        if seqs.start_q.numel() != self.batch + 1:
            raise ValueError("the plan must be of the cache's %d sequences" % self.batch)
        start = seqs.start_q
        more = start[1:] - start[:-1]
        longest = self._longest + seqs.max_q
        if longest > self.capacity and self.batch and not (k.is_cuda and torch.cuda.is_current_stream_capturing()):
            longest = int((self.used + more).max())  # waits for the device, which few calls have to
            if longest > self.capacity:
                raise ValueError("a sequence has more rows than the cache's capacity of %d" % self.capacity)
        self._longest = min(longest, self.capacity)
        row = torch.arange(k.shape[0], dtype=torch.int32, device=k.device)
        of = torch.searchsorted(start, row, right=True)
        base = self._base[1:-1]
        torch.add(self.start[:-1], self.used, out=base)
        base -= start[:-1]
        at = self._base[of] + row
        at = torch.where(at < self._end[of], at, self.batch * self.capacity).long()
        self._k.index_copy_(0, at, k)
        self._v.index_copy_(0, at, v)
        self.used += more
        self.used.clamp_(max=self.capacity)
        return Packed(start, self.start, seqs.max_q, self.capacity, self.used)


class MemoryBlock(torch.nn.Module):
    """rotary: positions by rotation (of the plan's pairs of every head) in place of the learned bias.  The state holds the
    rotation whole (turns, and rotation: layout and magnitude), so that a loaded one takes the place of the constructor's."""

    def __init__(self, w: int, heads: int, K: Sequence[int], kv_heads: Optional[int] = None, causal: bool = False,
                 buckets: int = 32, reach: int = 128, eps: float = 1e-5, table_dtype=torch.bfloat16,
                 dtype=torch.float32, device="cuda", memory: Optional[MemorySubnetwork] = None, rotary: Optional[Rotary] = None):
        super().__init__()
        kv_heads = heads if kv_heads is None else kv_heads
        if w % heads or heads % kv_heads:
            raise ValueError("w must be a multiple of heads, and heads of kv_heads")
        if w // heads not in HEAD_DIMS:
            raise ValueError("w / heads must be 32, 64 or 128")
        refusal = bias_refusal(heads, kv_heads, w // heads, dtype, buckets, reach) if rotary is None else None
        if refusal:
            raise ValueError(refusal)
        if heads > 64 * kv_heads:
            raise ValueError("heads must be at most 64 times kv_heads")
        if rotary is not None:
            if rotary.turns.dtype != torch.int64 or rotary.turns.dim() != 1:
                raise ValueError("a rotation's turns must be [pairs] int64")
            if not 1 <= rotary.turns.numel() <= w // heads // 2:
                raise ValueError("a rotation has 1 to head_dim / 2 pairs")
            if not math.isfinite(rotary.magnitude):
                raise ValueError("a rotation's magnitude must be finite")
        self.heads, self.kv_heads, self.head_dim, self.causal, self.eps = heads, kv_heads, w // heads, causal, eps
        new = dict(device=device, dtype=dtype)
        self.qkv = torch.nn.Linear(w, (heads + 2 * kv_heads) * self.head_dim, **new)
        self.proj = torch.nn.Linear(w, w, **new)
        self.rotates = rotary is not None
        if rotary is not None:
            self.register_buffer("turns", rotary.turns.to(device).clone())  # its own: a loaded state replaces it
            self.interleaved, self.magnitude = rotary.interleaved, rotary.magnitude
        else:
            self.bias = torch.nn.Parameter(torch.zeros((heads, buckets), **new))
            self.register_buffer("bucket", relative_buckets(buckets, reach, both=not causal, device=device))
        self.norm_w = torch.nn.ParameterList([torch.ones(w, **new) for _ in range(2)])
        self.norm_b = torch.nn.ParameterList([torch.zeros(w, **new) for _ in range(2)])
        self.memory = memory if memory is not None else MemorySubnetwork(w, K, table_dtype, dtype, device=device)

    def _save_to_state_dict(self, destination, prefix, keep_vars):
        super()._save_to_state_dict(destination, prefix, keep_vars)
        if self.rotates:  # with turns, the whole rotation
            destination[prefix + "rotation"] = torch.tensor([float(self.interleaved), self.magnitude], dtype=torch.float64)

    def _load_from_state_dict(self, state_dict, prefix, local_metadata, strict, missing_keys, unexpected_keys, error_msgs):
        own = self.turns.clone() if self.rotates else None
        super()._load_from_state_dict(state_dict, prefix, local_metadata, strict, missing_keys, unexpected_keys, error_msgs)
        if not self.rotates:
            return
        name, turns = prefix + "rotation", state_dict.get(prefix + "turns")
        rest = state_dict.get(name)
        if name in unexpected_keys:
            unexpected_keys.remove(name)
        if rest is not None and rest.shape != (2,):
            error_msgs.append("%s must hold a rotation's layout and magnitude" % name)
        elif rest is not None and turns is not None and turns.shape == own.shape:
            self.interleaved, self.magnitude = bool(rest[0]), float(rest[1])
        elif strict:
            # turns alone go with the block's layout and magnitude only where they are the block's own, to what a double rounds
            off = None if turns is None or turns.shape != own.shape or own.is_meta else turns.to(own.device) - own
            if off is None or not bool(((off < 1 << 14) & (off > -(1 << 14))).all()):
                missing_keys.append(name)

    def _heads(self, x: torch.Tensor):
        a, b = self.heads * self.head_dim, (self.heads + self.kv_heads) * self.head_dim
        x = self.qkv(x)
        return (x[:, :a].unflatten(1, (self.heads, self.head_dim)), x[:, a:b].unflatten(1, (self.kv_heads, self.head_dim)),
                x[:, b:].unflatten(1, (self.kv_heads, self.head_dim)))

    def _positions(self):
        """(rotation, bias), one of them None."""
        if self.rotates:
            return Rotary(self.turns, self.interleaved, self.magnitude), None
        return None, RelativeBias(self.bias, self.bucket)

    def _rest(self, a: torch.Tensor, x: torch.Tensor) -> torch.Tensor:
        x, _ = layer_norm(self.proj(a.flatten(1)), self.norm_w[0], self.norm_b[0], self.eps, residual=x)
        x, _ = layer_norm(self.memory(x), self.norm_w[1], self.norm_b[1], self.eps, residual=x)
        return x

    def forward(self, x: torch.Tensor, seqs: Packed, position: Optional[torch.Tensor] = None) -> torch.Tensor:
        """x [rows, w], its sequences packed by seqs; position (of a rotation): ``packed_positions`` of them by default, which
        several layers can share."""
        q, k, v = self._heads(x)
        plan, rel = self._positions()
        if plan is not None:
            q, k = rotate(q, k, packed_positions(seqs, x.shape[0]) if position is None else position, plan)
        return self._rest(attention(q, k, v, seqs, self.causal, rel=rel), x)

    @torch.no_grad()
    def serve(self, x: torch.Tensor, seqs: Packed, cache: Union[KeyValueCache, PagedCache], layer: int = 0) -> torch.Tensor:
        """The next rows of every sequence (whole prompts, pieces of them or single tokens; causal layers): their keys and
        values join the cache, and they attend over all of it.  A ``KeyValueCache`` is the layer's own; of a ``PagedCache`` it is
        layer ``layer``, seqs is what ``cache.extend`` returned for the step, and keys gather weights where the cache has them."""
        if not self.causal:
            raise ValueError("only a causal layer can be served piece by piece")
        q, k, v = self._heads(x)
        plan, rel = self._positions()
        if isinstance(cache, PagedCache):
            keys = cache.keys[layer]
            q = paged_append(k, v, keys, cache.table, seqs, q=q, rotary=plan)
            return self._rest(paged_attention(q, keys, cache.table, seqs, rel=rel, weigh=keys.weight is not None), x)
        if plan is not None:
            q, k = rotary_forward(q, k, packed_positions(seqs, x.shape[0], cache.used), plan)
        seqs = cache.append(k, v, seqs)
        return self._rest(attention_forward(q, cache.k, cache.v, seqs, True, rel=rel)[0], x)
