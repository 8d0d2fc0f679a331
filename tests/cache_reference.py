"""Plain 64-bit forms of rotary positions, of the cache in pages, of attention over it and of eviction from it, and how far a
computation that follows include/lram_cache.h may be from them.

With u the half unit of the results' type, r that of the operands' type (0 in fp32) and e = 2^-24:
  rotation   the angle, at most 1/8 turn from a quarter, is rounded three times (3 pi / 4 e < 2.4 e) and cut at 2^-32 of a turn
             (< 0.03 e); sine and cosine: five sums and products of terms below 1, then the magnitude: together below 10 e m;
             two products and a sum: 2 e;  so u |y| + 12 e m (|x1| + |x2|)
  scores     dz = (D + 8) e scale sum |q k| + 8 e (|z| + |bias|)
  out        u |out| + (r + dp + (n + 16) e) sum p |v|, dp = 2 max dz + 16 e the relative error of p
  weight     sum over queries and heads of p (dp + 16 e), and (columns + 8) e of the sum
"""
import math

import numpy as np
import torch

from layer_reference import E, HALF, half_operand


def angles(turns, position):
    """[rows, pairs] in radians, 64 bits: 2 pi frac(position turns / 2^64), the fraction in whole numbers."""
    t = np.array(turns.cpu().tolist(), dtype=object)
    out = np.empty((len(position), len(t)))
    for i, p in enumerate(position.cpu().tolist()):
        out[i] = [float((int(u) * p) % (1 << 64)) * 2.0 ** -64 for u in t]
    return torch.from_numpy(out * 2 * math.pi).to(turns.device)


def rotated(x, position, turns, interleaved, magnitude, backward=False):
    """(value, bound) of x [rows, heads, D] rotated."""
    n = turns.numel()
    a = angles(turns, position)[:, None]
    c, s = magnitude * torch.cos(a), magnitude * torch.sin(a) * (-1 if backward else 1)
    y, bound = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    x1, x2 = y[..., first].clone(), y[..., second].clone()
    y[..., first], y[..., second] = x1 * c - x2 * s, x1 * s + x2 * c
    size = 12 * E * abs(magnitude) * (x1.abs() + x2.abs())
    bound[..., first] = size + HALF[x.dtype] * y[..., first].abs()
    bound[..., second] = size + HALF[x.dtype] * y[..., second].abs()
    return y, bound


class Store:
    """A pool's contents key by key: k, v [pages, slot, head, D], position, weight [pages, slot, head], by the layout that the
    header states, with Python's own index arithmetic."""

    def __init__(self, keys):
        pages, heads, page = keys.position.shape
        e = keys.k.shape[5]
        dim = keys.k.shape[3] * e
        t, d = torch.arange(page)[:, None], torch.arange(dim)[None]
        k_at = ((t // 16 * (dim // e) + d // e) * 16 + t % 16) * e + d % e
        v_at = ((t // (4 * e) * (dim // 16) + d // 16) * 4 + t % 16 // 4) * 16 * e + d % 16 * e + t % (4 * e) // 16 * 4 + t % 4
        self.k_at, self.v_at = k_at.to(keys.k.device), v_at.to(keys.k.device)
        self.keys, self.page = keys, page
        flat = lambda x, at: x.reshape(pages, heads, -1)[:, :, at.flatten().to(x.device)].unflatten(2, at.shape).transpose(1, 2)  # noqa: E731
        self.k, self.v = flat(keys.k, self.k_at).clone(), flat(keys.v, self.v_at).clone()
        self.position = keys.position.transpose(1, 2).clone()
        self.weight = None if keys.weight is None else keys.weight.transpose(1, 2).clone()

    def write(self):
        """Back into the pool."""
        pages, heads, _ = self.keys.position.shape
        for x, at, mine in ((self.keys.k, self.k_at, self.k), (self.keys.v, self.v_at, self.v)):
            x.view(pages, heads, -1)[:, :, at.flatten()] = mine.transpose(1, 2).flatten(2)
        self.keys.position.copy_(self.position.transpose(1, 2))
        if self.weight is not None:
            self.keys.weight.copy_(self.weight.transpose(1, 2))

    def places(self, row, n):
        """(page, slot in it) of a sequence's key slots 0 ... n - 1; page -1 where there is none."""
        row = row.cpu()
        slot = torch.arange(min(n, row.numel() * self.page))
        page = row[slot // self.page].long()
        page[(page < 0) | (page >= self.k.shape[0])] = -1
        return page.to(self.k.device), (slot % self.page).to(self.k.device)


def attention(store, q, table, used, seen, start, scale, weight=None, bucket=None):
    """({"out": (value, bound)}, gathered [pages, slot, head], its bound) of new rows over the cache."""
    dt, (rows, hq, d) = q.dtype, q.shape
    hk = store.k.shape[2]
    group, u, r = hq // hk, HALF[dt], half_operand(dt)
    f64 = dict(dtype=torch.float64, device=q.device)
    out, bound = torch.zeros(q.shape, **f64), torch.zeros(q.shape, **f64)
    more = torch.zeros(store.position.shape, **f64)
    more_bound = torch.zeros_like(more)
    reach = 0 if bucket is None else bucket.numel() // 2
    for b in range(len(used)):
        q0, m = start[b], start[b + 1] - start[b]
        page, slot = store.places(table[b], used[b])
        page, slot = page[page >= 0], slot[page >= 0]
        n = page.numel()
        if m == 0 or n == 0:
            continue
        k = store.k[page, slot].double().transpose(0, 1).repeat_interleave(group, 0)  # [hq, n, d]
        v = store.v[page, slot].double().transpose(0, 1).repeat_interleave(group, 0)
        at = store.position[page, slot].long().t().repeat_interleave(group, 0)         # [hq, n]
        far = at[:, None] - (seen[b] - m + torch.arange(m, device=q.device))[None, :, None]
        shown = far <= 0
        x = q[q0:q0 + m].double().transpose(0, 1)
        z = x @ k.transpose(1, 2) * scale
        dz = (d + 8) * E * scale * (x.abs() @ k.abs().transpose(1, 2)) + 8 * E * z.abs()
        if weight is not None:
            of = bucket.long()[far.clamp(-reach, reach) + reach]
            bias = weight.double()[torch.arange(hq, device=q.device)[:, None, None], of]
            z, dz = z + bias, dz + 8 * E * torch.where(torch.isfinite(bias), bias.abs(), 0)
        z, dz = z.masked_fill(~shown, -math.inf), dz.masked_fill(~shown, 0.0)
        none = torch.isneginf(z).all(2, keepdim=True)
        p = torch.softmax(z.masked_fill(none, 0.0), 2).masked_fill(none, 0.0)
        dp = 2 * dz.amax(2, keepdim=True) + 16 * E
        o = p @ v
        out[q0:q0 + m] = o.transpose(0, 1)
        bound[q0:q0 + m] = (u * o.abs() + (r + dp + (n + 16) * E) * (p @ v.abs())).transpose(0, 1)
        got = p.unflatten(0, (hk, group)).sum((1, 2))
        more[page, slot] += got.t()
        more_bound[page, slot] += ((p * (dp + (n + 16) * E)).unflatten(0, (hk, group)).sum((1, 2)) + (m * group + 8) * E * got).t()
    return {"out": (out, bound)}, more, more_bound


def evicted(store, table, used, seen, budget, recent):
    """Cuts the store's sequences down to the budget, in place."""
    for b, n in enumerate(used):
        page, slot = store.places(table[b], n)
        n = page.numel()
        if n <= budget:
            continue
        p, s = page.cpu().numpy(), slot.cpu().numpy()
        for h in range(store.k.shape[2]):
            at = store.position[page, slot, h].cpu().numpy().astype(np.int64)
            w = store.weight[page, slot, h].cpu().numpy().astype(np.float64)
            newest = at >= seen[b] - recent
            # newest first, then by falling weight (NaN last), then by position, then by slot
            order = np.lexsort((at, np.where(newest, 0.0, np.where(np.isnan(w), np.inf, -w)),
                                np.where(newest, False, np.isnan(w)), ~newest))
            stays = np.zeros(n, bool)
            stays[order[:budget]] = True
            of, to = np.nonzero(stays[budget:])[0] + budget, np.nonzero(~stays[:budget])[0]
            for x in (store.k, store.v, store.position, store.weight):
                x[p[to], s[to], h] = x[p[of], s[of], h].clone()


def check(got, want, what=""):
    value, bound = want
    off = (got.double() - value).abs() - bound
    assert torch.isfinite(got).all(), what
    assert (off <= 0).all(), "%s: over its bound by %g (%g)" % (what, off.max(), (got.double() - value).abs().max())
