"""A transformer layer whose feed-forward part is the lattice memory (Sec. 3.1, 3.2: the memory subnetwork replaces the
dense feed-forward part of one layer of a BERT-style model).

    a = attention(x);  x = norm(x + a);  x = norm(x + memory(x))

over packed sequences of different lengths, in both directions or causal, with a learned relative position bias.  The
attention, its bias, the norms with their residual adds and the lookup run in liblram's kernels; the projections are
library GEMMs.
"""
from __future__ import annotations

from typing import Optional, Sequence

import torch

from .layer import Packed, RelativeBias, attention, attention_forward, layer_norm, layer_norm_forward, relative_buckets
from .memory_layer import MemorySubnetwork


class KeyValueCache:
    """Keys and values of ``batch`` sequences, ``capacity`` rows each; ``used`` [batch] int32 counts the rows in use.  The
    caller keeps a sequence's length within the capacity."""

    def __init__(self, batch: int, capacity: int, kv_heads: int, head_dim: int, dtype=torch.bfloat16, device="cuda"):
        self.batch, self.capacity = batch, capacity
        self.k = torch.empty((batch * capacity, kv_heads, head_dim), dtype=dtype, device=device)
        self.v = torch.empty_like(self.k)
        self.used = torch.zeros(batch, dtype=torch.int32, device=device)
        self.start = torch.arange(batch + 1, dtype=torch.int32, device=device) * capacity

    def append(self, k: torch.Tensor, v: torch.Tensor, seqs: Packed) -> Packed:
        """Adds the rows of k and v (packed by seqs.start_q) to their sequences; the plan of attention over the cache."""
        rows = k.shape[0]
        more = seqs.start_q[1:] - seqs.start_q[:-1]
        of = torch.repeat_interleave(torch.arange(self.batch, device=k.device), more.long(), output_size=rows)
        at = (self.start[:-1] + self.used - seqs.start_q[:-1])[of] + torch.arange(rows, device=k.device)
        self.k.index_copy_(0, at, k)
        self.v.index_copy_(0, at, v)
        self.used += more
        return Packed(seqs.start_q, self.start, seqs.max_q, self.capacity, self.used)


class MemoryBlock(torch.nn.Module):
    def __init__(self, w: int, heads: int, K: Sequence[int], kv_heads: Optional[int] = None, causal: bool = False,
                 buckets: int = 32, reach: int = 128, eps: float = 1e-5, table_dtype=torch.bfloat16,
                 dtype=torch.float32, device="cuda", memory: Optional[MemorySubnetwork] = None):
        super().__init__()
        kv_heads = heads if kv_heads is None else kv_heads
        if w % heads or heads % kv_heads:
            raise ValueError("w must be a multiple of heads, and heads of kv_heads")
        self.heads, self.kv_heads, self.head_dim, self.causal, self.eps = heads, kv_heads, w // heads, causal, eps
        new = dict(device=device, dtype=dtype)
        self.qkv = torch.nn.Linear(w, (heads + 2 * kv_heads) * self.head_dim, **new)
        self.proj = torch.nn.Linear(w, w, **new)
        self.bias = torch.nn.Parameter(torch.zeros((heads, buckets), **new))
        self.register_buffer("bucket", relative_buckets(buckets, reach, both=not causal, device=device))
        self.norm_w = torch.nn.ParameterList([torch.ones(w, **new) for _ in range(2)])
        self.norm_b = torch.nn.ParameterList([torch.zeros(w, **new) for _ in range(2)])
        self.memory = memory if memory is not None else MemorySubnetwork(w, K, table_dtype, dtype, device=device)

    def _heads(self, x: torch.Tensor):
        a, b = self.heads * self.head_dim, (self.heads + self.kv_heads) * self.head_dim
        x = self.qkv(x)
        return (x[:, :a].unflatten(1, (self.heads, self.head_dim)), x[:, a:b].unflatten(1, (self.kv_heads, self.head_dim)),
                x[:, b:].unflatten(1, (self.kv_heads, self.head_dim)))

    def forward(self, x: torch.Tensor, seqs: Packed) -> torch.Tensor:
        """x [rows, w], its sequences packed by seqs."""
        q, k, v = self._heads(x)
        a = attention(q, k, v, seqs, self.causal, rel=RelativeBias(self.bias, self.bucket))
        x, _ = layer_norm(self.proj(a.flatten(1)), self.norm_w[0], self.norm_b[0], self.eps, residual=x)
        x, _ = layer_norm(self.memory(x), self.norm_w[1], self.norm_b[1], self.eps, residual=x)
        return x

    @torch.no_grad()
    def serve(self, x: torch.Tensor, seqs: Packed, cache: KeyValueCache) -> torch.Tensor:
        """The next rows of every sequence (whole prompts, pieces of them or single tokens; causal layers): their keys and
        values join the cache, and they attend over all of it."""
        if not self.causal:
            raise ValueError("only a causal layer can be served piece by piece")
        q, k, v = self._heads(x)
        seqs = cache.append(k, v, seqs)
        a, _ = attention_forward(q, cache.k, cache.v, seqs, True, rel=RelativeBias(self.bias, self.bucket))
        x, _, _, _ = layer_norm_forward(self.proj(a.flatten(1)), self.norm_w[0], self.norm_b[0], self.eps, residual=x)
        x, _, _, _ = layer_norm_forward(self.memory(x).contiguous(), self.norm_w[1], self.norm_b[1], self.eps, residual=x)
        return x
