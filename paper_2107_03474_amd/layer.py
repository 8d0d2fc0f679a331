"""The operators around the lattice memory in a transformer layer: layer norm (with the residual add in front of it),
attention over packed sequences, and the learned relative position bias inside it.

As in the package's other calls, this module only marshals torch tensors and the current HIP stream into the C ABI
(``include/lram_layer.h``); the work is done by the library's HIP kernels, and there is no fallback.  Sums, statistics and
partial results are fp32, and results and gradients come in their inputs' types, rounded once from it.  In bf16 attention's
softmax weights and their gradient are rounded as well, where they enter a product of the matrix cores.
"""
from __future__ import annotations

import ctypes
import math
from typing import NamedTuple, Optional, Sequence, Tuple

import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable

from . import BF16, F32, LramError, _dev
from . import load as _load_library

__all__ = ["layer_norm_forward", "layer_norm_backward", "layer_norm", "Packed", "pack", "RelativeBias",
           "relative_buckets", "AttentionSaved", "attention_forward", "attention_backward", "attention"]

_P, _I64, _I32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32


class _Attention(ctypes.Structure):
    """lram_attention"""
    _fields_ = ([(n, _I32) for n in ("dtype", "wdtype", "heads", "kv_heads", "head_dim", "batch", "causal")] +
                [("scale", ctypes.c_float)] + [(n, _I64) for n in ("tq", "tk", "max_q", "max_k")] +
                [(n, _P) for n in ("q", "k", "v")] +
                [(n, _I64) for n in ("q_row", "q_head", "k_row", "k_head", "v_row", "v_head")] +
                [(n, _P) for n in ("start_q", "start_k", "used_k", "rel_weight", "rel_bucket")] +
                [("rel_buckets", _I32), ("rel_reach", _I32)])


_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = _load_library()
        I, SZ, SZP = ctypes.c_int, ctypes.c_size_t, ctypes.POINTER(ctypes.c_size_t)
        A = ctypes.POINTER(_Attention)
        lib.lram_layer_last_hip_error.restype = I
        lib.lram_layer_norm_forward.argtypes = [_P, _P, _P, _P, I, I, _I64, _I64, ctypes.c_double, _P, _P, _P, _P, _P]
        lib.lram_layer_norm_backward_workspace_bytes.argtypes = [_I64, _I64, I, SZP]
        lib.lram_layer_norm_backward.argtypes = [_P, _P, _P, _P, _P, _P, I, I, _I64, _I64, _P, _P, _P, _P, SZ, _P]
        lib.lram_attention_forward_workspace_bytes.argtypes = [A, SZP]
        lib.lram_attention_forward.argtypes = [A, _P, _P, _P, _P, SZ, _P]
        lib.lram_attention_backward_workspace_bytes.argtypes = [A, SZP]
        lib.lram_attention_backward.argtypes = [A, _P, _P, _P, _P, _P, _P, _P, _P, _P, SZ, _P]
        _lib = lib
    return _lib


def _check(rc: int):
    if rc != 0:
        lib = _library()
        msg = lib.lram_strerror(rc).decode()
        if rc == 6:
            msg += " (hipError %d)" % lib.lram_layer_last_hip_error()
        raise LramError(msg)


def _type(t: torch.Tensor, name: str) -> int:
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise LramError("%s must be float32 or bfloat16" % name)


# Small calls are bound by what happens on the host, so the checks below come cheapest first.

def _stream(device: torch.device) -> int:
    """The current stream of the device (the raw handle: torch's stream object costs 2 us to make)."""
    return torch._C._cuda_getCurrentRawStream(device.index)


def _ptr(t: torch.Tensor, name: str, dtype: torch.dtype, shape, like: torch.Tensor) -> int:
    """Device address of a contiguous tensor of this type and shape on like's device."""
    if not (t.dtype is dtype and t.shape == shape and t.device == like.device and t.is_contiguous() and t.is_cuda):
        _dev(t, name, dtype, shape, like=like)  # says what is wrong
    return t.data_ptr()


def _moved(t: torch.Tensor):
    """(address, copy) of a contiguous tensor that does not start on 16 bytes, as the kernels want it: later rows of an odd
    width, among them the gradients that torch.cat hands on."""
    t = t.clone()
    return t.data_ptr(), t


def _scratch(nbytes: int, workspace: Optional[torch.Tensor], like: torch.Tensor):
    """(pointer, bytes, tensor to keep until the launch) of a call's workspace."""
    if workspace is None:
        if not nbytes:
            return None, 0, None
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=like.device)
        return workspace.data_ptr(), nbytes, workspace
    return _dev(workspace, "workspace", like=like), workspace.numel() * workspace.element_size(), workspace


def _records(*inputs: Optional[torch.Tensor]) -> bool:
    """Whether autograd follows a call with these inputs (forward mode, which the wrappers refuse, among it: a tensor that
    carries a tangent shows it only to them)."""
    return (forward_ad._current_level >= 0 or
            torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in inputs))


# ---------------------------------------------------------------------------
# Layer norm.

def _norm_args(x: torch.Tensor, weight: torch.Tensor, name: str):
    if x.dim() < 1:
        raise LramError("%s must be [..., width]" % name)
    if not (x.is_cuda and x.is_contiguous()):
        _dev(x, name)
    width = x.shape[-1]
    if weight.dtype is not x.dtype and weight.dtype is not torch.float32:
        raise LramError("weight must be float32 or of %s's type" % name)
    return x.numel() // width if width else 0, width, _type(x, name), _type(weight, "weight")


def layer_norm_forward(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor, eps: float = 1e-5,
                       residual: Optional[torch.Tensor] = None, save: bool = True):
    """(y, h, mean, rstd): h = x + residual in x's type (x itself without a residual), y its layer norm over the last
    dimension, and the rows' statistics (fp32 [...]) for the backward, None without ``save``."""
    lib = _library()
    rows, width, dt, wt = _norm_args(x, weight, "x")
    wp = _ptr(weight, "weight", weight.dtype, (width,), x)
    bp = _ptr(bias, "bias", weight.dtype, (width,), x)
    xp = x.data_ptr()
    if xp & 15:
        xp, x = _moved(x)
    rp = hp = None
    h = x
    if residual is not None:
        rp = _ptr(residual, "residual", x.dtype, x.shape, x)
        if rp & 15:
            rp, residual = _moved(residual)
        h = torch.empty_like(x)
        hp = h.data_ptr()
    y = torch.empty_like(x)
    mean = rstd = mp = sp = None
    if save:
        mean = x.new_empty(x.shape[:-1], dtype=torch.float32)
        rstd = torch.empty_like(mean)
        mp, sp = mean.data_ptr(), rstd.data_ptr()
    rc = lib.lram_layer_norm_forward(xp, rp, wp, bp, dt, wt, rows, width, eps, hp, y.data_ptr(), mp, sp,
                                     _stream(x.device))
    if rc:
        if not 1 <= width <= 16384:
            raise LramError("rows must have 1 to 16384 elements")
        if not eps >= 0:
            raise LramError("eps must not be negative")
        _check(rc)
    return y, h, mean, rstd


def layer_norm_backward(h: torch.Tensor, weight: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                        grad_y: torch.Tensor, grad_h: Optional[torch.Tensor] = None, want_grad_weight: bool = True,
                        workspace: Optional[torch.Tensor] = None):
    """(grad_x, grad_weight, grad_bias) from what ``layer_norm_forward`` returned.  grad_h: the gradient that reaches h
    besides (the residual stream's); grad_x is that of x and of residual alike.  The weights' are None unless
    want_grad_weight."""
    lib = _library()
    rows, width, dt, wt = _norm_args(h, weight, "h")
    f32, lead = torch.float32, h.shape[:-1]
    wp = _ptr(weight, "weight", weight.dtype, (width,), h)
    mp, sp = _ptr(mean, "mean", f32, lead, h), _ptr(rstd, "rstd", f32, lead, h)
    yp = _ptr(grad_y, "grad_y", h.dtype, h.shape, h)
    gp = None if grad_h is None else _ptr(grad_h, "grad_h", h.dtype, h.shape, h)
    hp = h.data_ptr()
    if yp & 15:
        yp, grad_y = _moved(grad_y)
    if gp is not None and gp & 15:
        gp, grad_h = _moved(grad_h)
    if hp & 15:
        hp, h = _moved(h)
    gx = torch.empty_like(h)
    gw = gb = gwp = gbp = ws = keep = None
    ws_bytes = 0
    if want_grad_weight:
        gw, gb = torch.empty_like(weight), torch.empty_like(weight)
        gwp, gbp = gw.data_ptr(), gb.data_ptr()
        n = ctypes.c_size_t(0)
        if workspace is None:
            _check(lib.lram_layer_norm_backward_workspace_bytes(rows, width, dt, ctypes.byref(n)))
        ws, ws_bytes, keep = _scratch(n.value, workspace, h)
    rc = lib.lram_layer_norm_backward(hp, wp, mp, sp, yp, gp, dt, wt, rows, width, gx.data_ptr(), gwp, gbp,
                                      ws, ws_bytes, _stream(h.device))
    del keep
    if rc:
        _check(rc)
    return gx, gw, gb


class LayerNorm(torch.autograd.Function):
    """Autograd wrapper: (y, h)."""

    @staticmethod
    def forward(ctx, x, residual, weight, bias, eps):
        x = x.contiguous()
        residual = None if residual is None else residual.contiguous()
        y, h, mean, rstd = layer_norm_forward(x, weight.contiguous(), bias.contiguous(), eps, residual)
        ctx.save_for_backward(h, weight.contiguous(), mean, rstd)
        ctx.residual = residual is not None
        ctx.set_materialize_grads(False)
        if residual is None:
            return y, None
        return y, h

    @staticmethod
    @once_differentiable
    def backward(ctx, gy, gh):
        h, weight, mean, rstd = ctx.saved_tensors
        if gy is None:
            return gh, gh if ctx.residual else None, None, None, None
        gx, gw, gb = layer_norm_backward(h, weight, mean, rstd, gy.contiguous(),
                                         None if gh is None else gh.contiguous(),
                                         want_grad_weight=ctx.needs_input_grad[2] or ctx.needs_input_grad[3])
        return gx, gx if ctx.residual else None, gw, gb, None


def layer_norm(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor, eps: float = 1e-5,
               residual: Optional[torch.Tensor] = None):
    """The layer norm of x, differentiable; with a residual (y, h): the norm of h = x + residual, and h."""
    if not _records(x, residual, weight, bias):
        y, h, _, _ = layer_norm_forward(x.contiguous(), weight.contiguous(), bias.contiguous(), float(eps),
                                        None if residual is None else residual.contiguous(), save=False)
    else:
        y, h = LayerNorm.apply(x, residual, weight, bias, float(eps))
    return y if residual is None else (y, h)


# ---------------------------------------------------------------------------
# Attention over packed sequences.

class Packed(NamedTuple):
    """Where a batch's sequences lie (int32 device tensors): sequence b has the rows start_q[b] ... start_q[b + 1] - 1 of
    q and start_k[b] ... start_k[b + 1] - 1 of k and v, of the latter only the first used_k[b] where used_k is given (a
    cache).  Rows before the first sequence and past the last one belong to none.  max_q and max_k: the longest expected; what
    exceeds them costs time, not results."""
    start_q: torch.Tensor
    start_k: torch.Tensor
    max_q: int
    max_k: int
    used_k: Optional[torch.Tensor] = None


def pack(queries: Sequence[int], keys: Optional[Sequence[int]] = None, capacity: int = 0, device="cuda") -> Packed:
    """The plan of sequences of these lengths, packed one after the other; keys: their keys' lengths (the queries' by
    default); capacity: rows that a cache holds for every sequence, of which ``keys`` are used."""
    keys = queries if keys is None else keys
    if len(queries) != len(keys) or any(n < 0 for n in queries) or any(n < 0 for n in keys):
        raise LramError("queries and keys must be lengths of the same sequences")
    if capacity and any(n > capacity for n in keys):
        raise LramError("a sequence has more keys than the cache holds for it")

    def starts(lengths):
        at = [0]
        for n in lengths:
            at.append(at[-1] + int(n))
        if at[-1] >= 1 << 31:
            raise LramError("2^31 rows or more")
        return torch.tensor(at, dtype=torch.int32).to(device)

    return Packed(starts(queries), starts([capacity] * len(keys) if capacity else keys), max(queries, default=0),
                  max(keys, default=0), torch.tensor(list(keys), dtype=torch.int32).to(device) if capacity else None)


class RelativeBias(NamedTuple):
    """Learned bias of a query-key pair by head and bucket of their distance: weight [heads, buckets] (q's type or
    fp32), bucket [2 reach + 1] int32 (``relative_buckets``): the bucket of key minus query = -reach ... reach, the ends
    aligned; longer distances take the last one's.  A weight of -inf hides its keys; finite ones from 1.2e7 on in
    magnitude, the type's lowest value among them, count alike, and no score matters beside them.  At most 256 buckets, and
    heads / kv_heads (2 reach + 193) at most 4096 (in fp32 with head_dim 128: 2 reach + 193 at most 1365)."""
    weight: torch.Tensor
    bucket: torch.Tensor


def relative_buckets(buckets: int, reach: int, both: bool = True, device="cuda") -> torch.Tensor:
    """Buckets of the distances -reach ... reach by T5's rule (Raffel et al., arXiv 1910.10683, Sec. 2.1): half of a side's
    one distance each, the others growing as powers up to reach; ``both``: half of the buckets for keys behind the query,
    else none (a key behind it counts as distance 0)."""
    side = buckets // 2 if both else buckets
    near = max(side // 2, 1)
    n = side - near
    if buckets < 1 or side < 1 or reach < near:
        raise LramError("relative_buckets needs buckets >= 1 (2 for both sides) and reach >= half of a side's buckets")

    def one(a):  # near + floor(log(a / near) / log(reach / near) n), at most side - 1, in whole numbers
        return a if a < near else near + sum(a ** n * near ** c >= near ** n * reach ** c for c in range(1, n))

    got = [min(one(abs(d) if both else max(-d, 0)), side - 1) + (side if both and d > 0 else 0)
           for d in range(-reach, reach + 1)]
    return torch.tensor(got, dtype=torch.int32).to(device)


class AttentionSaved(NamedTuple):
    """What ``attention_backward`` needs beside the result: lse [rows, heads] fp32 (log2 of the softmax sums) and, bf16,
    the part of the result that its rounding left out."""
    lse: torch.Tensor
    residue: Optional[torch.Tensor]


def _heads(t: torch.Tensor, name: str, like: torch.Tensor):
    """(address, row stride, head stride) of a [rows, heads, head_dim] tensor whose last dimension is dense."""
    shape = t.shape
    if len(shape) != 3:
        raise LramError("%s must be [rows, heads, head_dim]" % name)
    if not t.is_cuda:
        raise LramError("%s must be a GPU tensor" % name)
    if t is not like and (t.dtype is not like.dtype or t.device != like.device or shape[2] != like.shape[2]):
        raise LramError("%s must have q's device, type and head_dim" % name)
    row, head, one = t.stride()
    if one != 1 and shape[2] > 1 and t.numel():
        raise LramError("%s must be dense along head_dim" % name)
    # a dimension of size 0 or 1 has no stride to speak of
    return (t.data_ptr(), row if shape[0] > 1 else shape[1] * shape[2], head if shape[1] > 1 else shape[2])


HEAD_DIMS = (32, 64, 128)


def bias_refusal(heads: int, kv_heads: int, head_dim: int, dtype: torch.dtype, buckets: int, reach: int) -> Optional[str]:
    """Why a relative bias of this size is not offered (its distances have to fit the kernels' LDS), None if it is."""
    if not 1 <= buckets <= 256:
        return "a relative bias has 1 to 256 buckets"
    if heads // kv_heads * (2 * reach + 193) > 4096:
        return "heads / kv_heads (2 reach + 193) must be at most 4096 with a relative bias"
    if dtype == torch.float32 and head_dim == 128 and 2 * reach + 193 > 1365:
        return "2 reach + 193 must be at most 1365 with a relative bias, float32 and head_dim 128"
    return None


def _check_attention(rc: int, a: _Attention):
    """Raises what the library refused, in the caller's terms where they can be told."""
    why = None
    if rc in (1, 3):  # argument, type
        per = 8 if a.dtype == BF16 else 4
        strides = (a.q_row, a.q_head, a.k_row, a.k_head, a.v_row, a.v_head)
        if a.head_dim not in HEAD_DIMS:
            why = "head_dim must be 32, 64 or 128"
        elif a.kv_heads < 1 or a.heads < 1 or a.heads % a.kv_heads or a.heads > 64 * a.kv_heads:
            why = "q's heads must be a multiple of k's, at most 64 times as many"
        elif not 0 < a.scale < math.inf:
            why = "scale must be positive and finite"
        elif any(p is not None and p % 16 for p in (a.q, a.k, a.v)) or any(s % per for s in strides) or any(
                not a.head_dim <= s <= 1 << 22 for s in strides[::2]):
            why = ("q, k and v must start on 16 bytes, with strides of whole 16 bytes and rows at least head_dim and at most "
                   "2^22 elements apart")
        elif a.rel_weight:
            why = bias_refusal(a.heads, a.kv_heads, a.head_dim, torch.float32 if a.dtype == F32 else torch.bfloat16,
                               a.rel_buckets, a.rel_reach)
    if why:
        raise LramError(why)
    _check(rc)


def _describe(q, k, v, seqs: Packed, causal, scale, rel: Optional[RelativeBias]):
    a = _Attention()
    a.q, a.q_row, a.q_head = _heads(q, "q", q)
    a.k, a.k_row, a.k_head = _heads(k, "k", q)
    a.v, a.v_row, a.v_head = _heads(v, "v", q)
    if k.shape != v.shape:
        raise LramError("k and v must have the same shape")
    a.tq, heads, dim = q.shape
    a.tk, a.kv_heads, _ = k.shape
    a.heads, a.head_dim = heads, dim
    batch = a.batch = seqs.start_q.numel() - 1
    if batch < 0:
        raise LramError("start_q must be [batch + 1]")
    i32 = torch.int32
    a.dtype = _type(q, "q")
    a.causal = 1 if causal else 0
    a.scale = 1.0 / math.sqrt(max(dim, 1)) if scale is None else scale
    a.max_q, a.max_k = seqs.max_q, seqs.max_k
    a.start_q = _ptr(seqs.start_q, "start_q", i32, (batch + 1,), q)
    a.start_k = _ptr(seqs.start_k, "start_k", i32, (batch + 1,), q)
    if seqs.used_k is not None:
        a.used_k = _ptr(seqs.used_k, "used_k", i32, (batch,), q)
    if rel is not None:
        w, bucket = rel
        if w.dim() != 2 or bucket.dim() != 1 or bucket.numel() % 2 != 1:
            raise LramError("a relative bias has weight [heads, buckets] and bucket [2 reach + 1]")
        if w.dtype is not q.dtype and w.dtype is not torch.float32:
            raise LramError("the relative bias's weight must be float32 or of q's type")
        buckets, n = w.shape[1], bucket.shape[0]
        a.rel_weight = _ptr(w, "rel.weight", w.dtype, (heads, buckets), q)
        a.rel_bucket = _ptr(bucket, "rel.bucket", i32, (n,), q)
        a.wdtype = _type(w, "rel.weight")
        a.rel_buckets, a.rel_reach = buckets, n // 2
    return a


def attention_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, seqs: Packed, causal: bool = False,
                      scale: Optional[float] = None, rel: Optional[RelativeBias] = None, save: bool = False,
                      workspace: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, Optional[AttentionSaved]]:
    """(out, saved): softmax(scale q k^T + bias) v of packed sequences, q [rows, heads, head_dim], k and v [rows, kv_heads,
    head_dim] (from 16 bytes on, with row and head strides of whole 16 bytes; head_dim 32, 64 or 128; scale 1 / sqrt(head_dim)
    by default).  The ends of a
    sequence's queries and keys are aligned, and ``causal`` queries see no key past theirs.  saved (with ``save``): for
    ``attention_backward``."""
    lib = _library()
    a = _describe(q, k, v, seqs, causal, scale, rel)
    out = q.new_empty(q.shape)
    saved = lse = residue = None
    if save:
        saved = AttentionSaved(q.new_empty(q.shape[:2], dtype=torch.float32),
                               torch.empty_like(out) if q.dtype is torch.bfloat16 else None)
        lse = saved.lse.data_ptr()
        residue = None if saved.residue is None else saved.residue.data_ptr()
    n = ctypes.c_size_t(0)
    if workspace is None:
        rc = lib.lram_attention_forward_workspace_bytes(a, n)
        if rc:
            _check_attention(rc, a)
    ws, ws_bytes, keep = _scratch(n.value, workspace, q)
    rc = lib.lram_attention_forward(a, out.data_ptr(), lse, residue, ws, ws_bytes, _stream(q.device))
    del keep
    if rc:
        _check_attention(rc, a)
    return out, saved


def attention_backward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, seqs: Packed, out: torch.Tensor,
                       saved: AttentionSaved, grad_out: torch.Tensor, causal: bool = False,
                       scale: Optional[float] = None, rel: Optional[RelativeBias] = None,
                       workspace: Optional[torch.Tensor] = None):
    """(grad_q, grad_k, grad_v, grad_rel) from what ``attention_forward`` returned (with ``save`` and the same
    arguments); grad_rel, of the bias's weight, is None without one.  Rows of k and v that no query may see get zeros."""
    lib = _library()
    a = _describe(q, k, v, seqs, causal, scale, rel)
    op = _ptr(out, "out", q.dtype, q.shape, q)
    gp = _ptr(grad_out, "grad_out", q.dtype, q.shape, q)
    if gp & 15:
        gp, grad_out = _moved(grad_out)
    lp = _ptr(saved.lse, "saved.lse", torch.float32, q.shape[:2], q)
    rp = None if saved.residue is None else _ptr(saved.residue, "saved.residue", q.dtype, q.shape, q)
    gq = torch.empty_like(out)
    gk = k.new_empty(k.shape)
    gv = torch.empty_like(gk)
    grel = None if rel is None else torch.empty_like(rel.weight)
    n = ctypes.c_size_t(0)
    if workspace is None:
        _check_attention(lib.lram_attention_backward_workspace_bytes(a, n), a)
    ws, ws_bytes, keep = _scratch(n.value, workspace, q)
    rc = lib.lram_attention_backward(a, op, rp, lp, gp, gq.data_ptr(), gk.data_ptr(), gv.data_ptr(),
                                     None if grel is None else grel.data_ptr(), ws, ws_bytes, _stream(q.device))
    del keep
    if rc:
        _check_attention(rc, a)
    return gq, gk, gv, grel


class Attention(torch.autograd.Function):
    """Autograd wrapper of attention over packed sequences."""

    @staticmethod
    def forward(ctx, q, k, v, weight, bucket, seqs, causal, scale):
        rel = None if weight is None else RelativeBias(weight.contiguous(), bucket)
        out, saved = attention_forward(q, k, v, seqs, causal, scale, rel, save=True)
        ctx.save_for_backward(q, k, v, out, saved.lse, saved.residue, None if rel is None else rel.weight, bucket,
                              seqs.start_q, seqs.start_k, seqs.used_k)
        ctx.rest = (seqs.max_q, seqs.max_k, causal, scale)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, g):
        q, k, v, out, lse, residue, weight, bucket, start_q, start_k, used_k = ctx.saved_tensors
        max_q, max_k, causal, scale = ctx.rest
        rel = None if weight is None else RelativeBias(weight, bucket)
        gq, gk, gv, grel = attention_backward(q, k, v, Packed(start_q, start_k, max_q, max_k, used_k), out,
                                              AttentionSaved(lse, residue), g.contiguous(), causal, scale, rel)
        return gq, gk, gv, grel, None, None, None, None


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, seqs: Packed, causal: bool = False,
              scale: Optional[float] = None, rel: Optional[RelativeBias] = None) -> torch.Tensor:
    """``attention_forward``'s result, differentiable in q, k, v and the bias's weight."""
    if not _records(q, k, v, None if rel is None else rel.weight):
        rel = None if rel is None else RelativeBias(rel.weight.contiguous(), rel.bucket)
        return attention_forward(q, k, v, seqs, causal, scale, rel)[0]  # nothing to be kept for a backward
    return Attention.apply(q, k, v, None if rel is None else rel.weight, None if rel is None else rel.bucket, seqs,
                           bool(causal), scale)
