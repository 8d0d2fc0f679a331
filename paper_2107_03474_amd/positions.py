"""Rotary positions for the attention of a layer around the lattice memory: the rotation of queries and keys by their places in
the text, forward and backward.

As in the package's other calls, this module only marshals torch tensors and the current HIP stream into the C ABI
(``include/lram_cache.h``); there is no fallback.  Angles of a plan's turns are exact to 2^-32 of a turn at any position, those
turns are its frequencies rounded to the nearest 2^-64 (2^-34 of a turn at the farthest position), and a rotated value is rounded
once.
"""
from __future__ import annotations

import ctypes
import decimal
import math
from typing import NamedTuple, Optional, Tuple

import torch
from torch.autograd.function import once_differentiable

from . import BF16, LramError
from . import load as _load_library
from .layer import Packed, _check, _heads, _ptr, _records, _type

__all__ = ["Rotary", "rotary_plan", "packed_positions", "rotary_forward", "rotary_backward", "rotary"]

_P, _I64, _I32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32


class _Rotary(ctypes.Structure):
    """lram_rotary"""
    _fields_ = [("pairs", _I32), ("interleaved", _I32), ("magnitude", ctypes.c_float), ("turns", _P)]


TWO_PI = decimal.Decimal("6.28318530717958647692528676655900576839433879875021164194988918461563"
                         "2812572417997256069650684234135964296173")
_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = _load_library()
        R, I = ctypes.POINTER(_Rotary), ctypes.c_int
        lib.lram_positions.argtypes = [_P, _P, _I32, _I64, _P, _P]
        lib.lram_rotate.argtypes = [R, I, I, _I64, _I32, _P, _P, _I64, _I64, _I32, _P, _P, _I64, _I64, _I32, _P, _P]
        _lib = lib
    return _lib


def _launch(device: torch.device, call, *args) -> int:
    """call(*args, the device's current stream), with the device as the current one."""
    if device.index == torch._C._cuda_getDevice():
        return call(*args, torch._C._cuda_getCurrentRawStream(device.index))
    with torch.cuda.device(device):
        return call(*args, torch._C._cuda_getCurrentRawStream(device.index))


class Rotary(NamedTuple):
    """Pair i of a head, (x[2i], x[2i + 1]) interleaved or (x[i], x[i + pairs]), turns by turns[i] / 2^64 of a full turn a token
    and is multiplied by magnitude; turns [pairs] int64 (the fraction's 64 bits).  Dimensions past 2 pairs stay."""
    turns: torch.Tensor
    interleaved: bool = False
    magnitude: float = 1.0


def rotary_plan(dim: int, base: float = 10000.0, interleaved: bool = False, scaling: Optional[str] = None, factor: float = 1.0,
                length: int = 0, low: float = 1.0, high: float = 32.0, device="cuda") -> Rotary:
    """The rotation of a head's first ``dim`` dimensions by base^(-2 i / dim) radians a token (Su et al., arXiv 2104.09864),
    for texts ``factor`` times as long as those of training with one of the scalings
      "linear"  every frequency divided by factor (Chen et al., arXiv 2306.15595)
      "base"    base times factor^(dim / (dim - 2)): the slowest frequency is divided by factor, the fastest stays
      "parts"   frequencies that turn at most ``low`` times over ``length`` tokens divided by factor, those of ``high`` turns
                and more kept, between them in proportion; magnitude 0.1 ln factor + 1 (Peng et al., arXiv 2309.00071)."""
    if dim < 2 or dim % 2 or not base > 0:
        raise LramError("rotary_plan needs an even number of dimensions and base > 0")
    if scaling not in (None, "linear", "base", "parts"):
        raise LramError("scaling must be None, 'linear', 'base' or 'parts'")
    if scaling and not (0 < factor < math.inf):
        raise LramError("factor must be positive and finite")
    if scaling == "parts" and not (length > 0 and 0 <= low < high):
        raise LramError("scaling 'parts' needs length > 0 and 0 <= low < high")
    if scaling == "base" and dim < 4:
        raise LramError("scaling 'base' needs at least 4 dimensions")
    magnitude = 0.1 * math.log(factor) + 1 if scaling == "parts" else 1.0
    # a double's 53 bits of a frequency would leave 2^-25 of a turn at the farthest positions, so decimal digits: 64 bits are 20,
    # and what is left holds whole turns
    with decimal.localcontext(decimal.Context(prec=100, rounding=decimal.ROUND_HALF_EVEN, traps=[])):
        def of(x):
            return decimal.Decimal(float(x))

        base, factor, size = of(base), of(factor) if scaling else None, decimal.Decimal(int(dim))
        if scaling == "base":
            base = base * factor ** (size / (size - 2))
        turns = [base ** (-2 * i / size) / TWO_PI for i in range(dim // 2)]
        if scaling == "linear":
            turns = [t / factor for t in turns]
        elif scaling == "parts":
            stays = [min(max((of(length) * t - of(low)) / (of(high) - of(low)), 0), 1) for t in turns]
            turns = [t * (s + (1 - s) / factor) for t, s in zip(turns, stays)]
        bits = [int((t * (1 << 64)).to_integral_value()) % (1 << 64) for t in turns]
    return Rotary(torch.tensor([b - (1 << 64) if b >> 63 else b for b in bits]).to(device), bool(interleaved), magnitude)


def packed_positions(seqs: Packed, rows: int, first: Optional[torch.Tensor] = None) -> torch.Tensor:
    """int32 [rows]: each row's place in its sequence (packed by seqs.start_q), counted from first [batch] (int32, zeros by
    default); 0 for rows of no sequence."""
    start = seqs.start_q
    batch = start.numel() - 1
    if batch < 0:
        raise LramError("start_q must be [batch + 1]")
    if not 0 <= rows <= 1 << 30:
        raise LramError("rows must be 0 to 2^30")
    i32 = torch.int32
    sp = _ptr(start, "start_q", i32, (batch + 1,), start)
    fp = None if first is None else _ptr(first, "first", i32, (batch,), start)
    at = start.new_empty(rows)
    rc = _launch(start.device, _library().lram_positions, sp, fp, batch, rows, at.data_ptr())
    if rc:
        _check(rc)
    return at


def _rotary(plan: Rotary, like: torch.Tensor) -> _Rotary:
    turns, interleaved, magnitude = plan
    n = turns.numel()
    if turns.dtype is torch.int64 and turns.dim() == 1 and turns.get_device() == like.get_device() and turns.is_contiguous():
        return _Rotary(n, 1 if interleaved else 0, magnitude, turns.data_ptr())
    return _Rotary(n, 1 if interleaved else 0, magnitude, _ptr(turns, "turns", torch.int64, (n,), like))  # says what is wrong


def _refusal(dtype, dim: int, plan: Rotary, tensors) -> Optional[str]:
    if dim % 8 or not 8 <= dim <= 1024:
        return "head_dim must be a multiple of 8, at most 1024"
    if not 1 <= plan.turns.numel() <= dim // 2:
        return "a rotation has 1 to head_dim / 2 pairs"
    if not math.isfinite(plan.magnitude):
        return "magnitude must be finite"
    per = 8 if dtype is torch.bfloat16 else 4
    for p, row, head in tensors:
        if p % 16 or row % per or head % per or not dim <= row <= 1 << 22 or head < 0:
            return ("queries and keys must start on 16 bytes, with strides of whole 16 bytes and rows at least head_dim and at "
                    "most 2^22 elements apart")
    return None


def _rotate(q, k, position, plan: Rotary, backward: bool):
    lib = _library()
    dt = _type(q, "q")
    places = [_heads(q, "q", q)]
    rows, heads, dim = q.shape
    if k is not None:
        places.append(_heads(k, "k", q))
        if k.shape[0] != rows:
            raise LramError("q and k must have the same rows")
    at = _ptr(position, "position", torch.int32, (rows,), q)
    r = _rotary(plan, q)
    # (new_empty takes half a microsecond longer)
    out_q = torch.empty_like(q, memory_format=torch.contiguous_format)
    out_k = None if k is None else torch.empty_like(k, memory_format=torch.contiguous_format)
    kv = 0 if k is None else k.shape[1]
    if not heads or k is not None and not kv:
        raise LramError("q and k must have heads")
    rc = _launch(q.device, lib.lram_rotate, r, dt, int(backward), rows, dim, at, *places[0], heads, out_q.data_ptr(),
                 *(places[1] if kv else (None, 0, 0)), kv, out_k.data_ptr() if kv else None)
    if rc:
        why = _refusal(q.dtype, dim, plan, places)
        if why:
            raise LramError(why)
        _check(rc)
    return out_q, out_k


def rotary_forward(q: torch.Tensor, k: Optional[torch.Tensor], position: torch.Tensor, plan: Rotary
                   ) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """(q, k) rotated: q [rows, heads, head_dim] and k [rows, kv_heads, head_dim] (or None) at the places position [rows] int32,
    which may be any.  They start on 16 bytes with strides of whole 16 bytes; head_dim is a multiple of 8, at most 1024."""
    return _rotate(q, k, position, plan, False)


def _as_heads(g: torch.Tensor) -> torch.Tensor:
    """A gradient as the kernel takes it: copied where its strides or its start do not fit."""
    per = 16 // g.element_size()
    row, head, one = g.stride()
    fits = one == 1 and row >= g.shape[2] and row % per == 0 and head % per == 0 and head >= 0 and row <= 1 << 22
    return g if fits and not g.data_ptr() % 16 else g.contiguous() if not g.is_contiguous() else g.clone()


def rotary_backward(grad_q: torch.Tensor, grad_k: Optional[torch.Tensor], position: torch.Tensor, plan: Rotary
                    ) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Gradients of ``rotary_forward``'s q and k from its results': the rotation the other way round."""
    if grad_q.dim() != 3 or grad_k is not None and grad_k.dim() != 3:
        raise LramError("gradients must be [rows, heads, head_dim]")
    return _rotate(_as_heads(grad_q), None if grad_k is None else _as_heads(grad_k), position, plan, True)


class Rotate(torch.autograd.Function):
    """Autograd wrapper of the rotation."""

    @staticmethod
    def forward(ctx, q, k, position, turns, interleaved, magnitude):
        ctx.save_for_backward(position, turns)
        ctx.rest = (interleaved, magnitude)
        ctx.set_materialize_grads(False)
        return rotary_forward(q, k, position, Rotary(turns, interleaved, magnitude))

    @staticmethod
    @once_differentiable
    def backward(ctx, gq, gk):
        position, turns = ctx.saved_tensors
        plan = Rotary(turns, *ctx.rest)
        gq, gk = gq if ctx.needs_input_grad[0] else None, gk if ctx.needs_input_grad[1] else None
        if gq is None and gk is None:
            return (None,) * 6
        if gq is None:
            return None, rotary_backward(gk, None, position, plan)[0], None, None, None, None
        gq, gk = rotary_backward(gq, gk, position, plan)
        return gq, gk, None, None, None, None


def rotary(q: torch.Tensor, k: Optional[torch.Tensor], position: torch.Tensor, plan: Rotary
           ) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """``rotary_forward``'s result, differentiable in q and k."""
    if not _records(q, k):
        return rotary_forward(q, k, position, plan)
    return Rotate.apply(q, k, position, plan.turns, bool(plan.interleaved), float(plan.magnitude))
