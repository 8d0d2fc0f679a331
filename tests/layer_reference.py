"""Plain 64-bit forms of the operators around the memory (layer norm, packed attention with its relative position bias)
with their gradients written out, and how far a computation that follows include/lram_layer.h may be from them.

The bounds follow the arithmetic that the header states: sums and softmax terms in fp32, the softmax's weights and ds
rounded to the operands' type before the products that use them, results rounded once.  With u the half unit of the
results' type, r that of the operands' type (0 in fp32, where nothing is rounded between), and e = 2^-24:
  z        n-term fp32 sums: |dz| <= (D + 8) e sum |q k| scale + 8 e |z|, through the row's maximum and lse twice
  p        relative error dp = 2 max dz + 16 e
  out      u |out| + (r + dp + n e) sum p |v|
  delta    sum |do| times out's bound before its rounding (2^-17 |out| is left when the residue is kept)
  ds       p (dp |do.v - delta| + (D + 8) e sum |do v| + ddelta) + r |ds|
and each gradient its own rounding plus these, summed over absolute values.
"""
import math

import torch

E = 2.0 ** -24
HALF = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16)}  # of a value rounded to nearest


def half_operand(dtype):
    return 0.0 if dtype == torch.float32 else HALF[dtype]


def norm(x, w, b, eps, residual=None, dy=None, dh=None):
    """{name: (value, bound)} of the norm and, with dy, its gradients; all inputs of their own types."""
    u, uw = HALF[x.dtype], HALF[w.dtype]
    x64 = x.double()
    got = {}
    if residual is not None:
        s = x64 + residual.double()
        got["h"] = (s, u * s.abs() + E * s.abs())
        x64 = (x.float() + residual.float()).to(x.dtype).double()  # what is returned is what is normed
    n = x64.shape[-1]
    mean = x64.mean(-1, keepdim=True)
    c = x64 - mean
    rstd = 1 / torch.sqrt((c * c).mean(-1, keepdim=True) + eps)
    xh = c * rstd
    # the mean's error moves every element alike; n-term sums in fp32 (a tree: 64 terms or fewer in line)
    dmean = 80 * E * x64.abs().mean(-1, keepdim=True)
    dxh = rstd * (dmean + 2 * E * x64.abs()) * (1 + 1e-3) + xh.abs() * (200 * E + rstd * dmean)
    w64, b64 = w.double(), b.double()
    y = xh * w64 + b64
    got["y"] = (y, u * y.abs() + dxh * w64.abs() + 4 * E * (xh * w64).abs() + E * y.abs())
    if dy is not None:
        g64 = dy.double()
        g = g64 * w64
        a, m = g.mean(-1, keepdim=True), (g * xh).mean(-1, keepdim=True)
        dx = rstd * (g - a - xh * m)
        da = 80 * E * g.abs().mean(-1, keepdim=True)
        dm = (g.abs() * dxh).mean(-1, keepdim=True) + 80 * E * (g * xh).abs().mean(-1, keepdim=True)
        ddx = rstd * (4 * E * g.abs() + da + dxh * m.abs() + xh.abs() * dm) + 200 * E * (
            rstd * (g.abs() + a.abs() + (xh * m).abs())) + rstd * rstd * dmean * dx.abs()
        if dh is not None:
            dx = dx + dh.double()
        got["dx"] = (dx, u * dx.abs() + ddx + 2 * E * dx.abs())
        rows = tuple(range(x64.dim() - 1))
        many = (x64[..., 0].numel() // 256 + 128) * E  # a register adds every 256th row at least, a tree the rest
        dw, db = (g64 * xh).sum(rows), g64.sum(rows)
        got["dw"] = (dw, uw * dw.abs() + (g64.abs() * dxh).sum(rows) + many * (g64 * xh).abs().sum(rows))
        got["db"] = (db, uw * db.abs() + many * g64.abs().sum(rows))
    return got


def attention(q, k, v, nq, nk, start_q, start_k, causal, scale, weight=None, bucket=None, do=None):
    """{name: (value, bound)} of packed attention over sequences of nq queries and nk keys that start at these rows."""
    dt, (tq, hq, d), hk = q.dtype, q.shape, k.shape[1]
    u, r, group = HALF[dt], half_operand(dt), hq // hk
    f64 = dict(dtype=torch.float64, device=q.device)
    got = {n: [torch.zeros(s, **f64), torch.zeros(s, **f64)] for n, s in
           (("out", q.shape), ("lse", q.shape[:2]), ("dq", q.shape), ("dk", k.shape), ("dv", k.shape))}
    got["lse"][0] += -math.inf
    if weight is not None:
        got["dw"] = [torch.zeros(weight.shape, **f64), torch.zeros(weight.shape, **f64)]
        reach = bucket.numel() // 2
    for m, n, q0, k0 in zip(nq, nk, start_q, start_k):
        if m == 0 or n == 0:
            continue
        far = torch.arange(n, device=q.device)[None] - torch.arange(m, device=q.device)[:, None] - (n - m)
        seen = far <= 0 if causal else torch.ones_like(far, dtype=torch.bool)
        q64 = q[q0:q0 + m].double().transpose(0, 1)                                     # [hq, m, d]
        k64, v64 = (t[k0:k0 + n].double().transpose(0, 1).repeat_interleave(group, 0) for t in (k, v))
        z = q64 @ k64.transpose(1, 2) * scale
        dz = (d + 8) * E * scale * (q64.abs() @ k64.abs().transpose(1, 2)) + 8 * E * z.abs()
        if weight is not None:
            of = bucket.long()[far.clamp(-reach, reach) + reach]
            bias = weight.double()[:, of]
            z, dz = z + bias, dz + 8 * E * bias.abs()
        z = z.masked_fill(~seen, -math.inf)
        dz = dz.masked_fill(~seen, 0.0)
        none = ~seen.any(1)                                                             # rows that see nothing
        lse = torch.logsumexp(z, 2)
        p = torch.exp(z - lse[..., None]).masked_fill(none[None, :, None], 0.0)
        worst = dz.amax(2, keepdim=True) + 16 * E
        dp = 2 * worst                                                                  # relative
        o = p @ v64
        raw = (r + dp + (n + 16) * E) * (p @ v64.abs())
        got["out"][0][q0:q0 + m] = o.transpose(0, 1)
        got["out"][1][q0:q0 + m] = (u * o.abs() + raw + E * o.abs()).transpose(0, 1)
        got["lse"][0][q0:q0 + m] = (lse / math.log(2)).transpose(0, 1)
        got["lse"][1][q0:q0 + m] = (2 * worst[..., 0] + (n + 16) * E + 4 * E * lse.abs().nan_to_num(0, 0, 0)).transpose(0, 1)
        if do is None:
            continue
        g64 = do[q0:q0 + m].double().transpose(0, 1)
        s = g64 @ v64.transpose(1, 2)
        delta = (g64 * o).sum(2, keepdim=True)
        ddelta = (g64.abs() * (raw + 2.0 ** -17 * o.abs())).sum(2, keepdim=True) + (d + 8) * E * (g64 * o).abs().sum(2, keepdim=True)
        ds = p * (s - delta)
        raw_ds = p * (dp * (s - delta).abs() + (d + 8) * E * (g64.abs() @ v64.abs().transpose(1, 2)) + ddelta) + 4 * E * ds.abs()
        dds = raw_ds + r * ds.abs()
        dq = scale * (ds @ k64)
        got["dq"][0][q0:q0 + m] = dq.transpose(0, 1)
        got["dq"][1][q0:q0 + m] = (u * dq.abs() + scale * ((dds + (n + 8) * E * ds.abs()) @ k64.abs())).transpose(0, 1)

        def shared(t):  # the heads of a group add up
            return t.unflatten(0, (hk, group)).sum(1).transpose(0, 1)

        many = (m * group + 16) * E
        dk, dv = scale * shared(ds.transpose(1, 2) @ q64), shared(p.transpose(1, 2) @ g64)
        got["dk"][0][k0:k0 + n] = dk
        got["dk"][1][k0:k0 + n] = u * dk.abs() + scale * shared((dds + many * ds.abs()).transpose(1, 2) @ q64.abs())
        got["dv"][0][k0:k0 + n] = dv
        got["dv"][1][k0:k0 + n] = u * dv.abs() + shared(((r + dp + many) * p).transpose(1, 2) @ g64.abs())
        if weight is not None:
            for c in range(weight.shape[1]):
                at = of == c
                got["dw"][0][:, c] += (ds * at).sum((1, 2))
                got["dw"][1][:, c] += ((raw_ds + many * ds.abs() + n * E * ds.abs()) * at).sum((1, 2))
    if weight is not None:
        got["dw"][1] += HALF[weight.dtype] * got["dw"][0].abs()
    return {n: tuple(t) for n, t in got.items()}


def assert_close(name, got, want):
    """got within its bound of the value everywhere (an equal infinity is equal)."""
    value, bound = want
    got = got.double().to(value.device)
    assert got.shape == value.shape, (name, got.shape, value.shape)
    off = torch.where(got == value, torch.zeros_like(value), (got - value).abs())
    bad = ~(off <= bound + 1e-30)
    if bool(bad.any()):
        i = int((off / (bound + 1e-30)).nan_to_num(math.inf).flatten().argmax())
        raise AssertionError("%s: %d of %d off, worst at %d: %r, exact %r, bound %.3g" % (
            name, int(bad.sum()), bad.numel(), i, float(got.flatten()[i]), float(value.flatten()[i]),
            float(bound.flatten()[i])))
