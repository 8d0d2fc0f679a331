"""Attention whose relative position bias has weights far from zero, against the 64-bit form and its derived bounds
(layer_reference.py)."""
import math

import pytest
import torch

import layer_reference as ref
import paper_2107_03474_amd as lram

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16
BOTH_TYPES = pytest.mark.parametrize("dtype", [F32, BF16])
BOTH_WAYS = pytest.mark.parametrize("causal", [False, True])


def _starts(n):
    return [sum(n[:i]) for i in range(len(n))]


def _inputs(lengths, hq, hk, d, dtype, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    tq = sum(lengths)
    q, do = (torch.randn((tq, hq, d), generator=g, device=DEV).to(dtype) for _ in range(2))
    k, v = (torch.randn((tq, hk, d), generator=g, device=DEV).to(dtype) for _ in range(2))
    return q, k, v, do


def _run(q, k, v, do, lengths, causal, w, bucket):
    seqs, rel = lram.pack(lengths), lram.RelativeBias(w, bucket)
    out, saved = lram.attention_forward(q, k, v, seqs, causal, rel=rel, save=True)
    dq, dk, dv, dw = lram.attention_backward(q, k, v, seqs, out, saved, do, causal, rel=rel)
    torch.cuda.synchronize()
    return dict(out=out, lse=saved.lse, dq=dq, dk=dk, dv=dv, dw=dw)


# ends inside a block of 32 rows, one row alone, tiles of several workgroups
LENGTHS = [[33], [200, 1, 65], [1, 31, 450]]


@BOTH_TYPES
@BOTH_WAYS
@pytest.mark.parametrize("shift", [100.0, -100.0, 300.0])
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
@pytest.mark.parametrize("reach", [3, 128])
def test_a_shift_of_every_weight(lengths, shift, reach, causal, dtype):
    """The softmax does not know a shift that all weights share; blocks past reach (3) and within it (128)."""
    q, k, v, do = _inputs(lengths, 4, 2, 64, dtype, 5)
    g = torch.Generator(device=DEV)
    g.manual_seed(6)
    w = (torch.randn((4, 8), generator=g, device=DEV) + shift).to(dtype)
    bucket = lram.relative_buckets(8, reach)
    got = _run(q, k, v, do, lengths, causal, w, bucket)
    want = ref.attention(q, k, v, lengths, lengths, _starts(lengths), _starts(lengths), causal, 0.125, w, bucket, do)
    for n, t in got.items():
        ref.assert_close(n, t, want[n])


def _by_autograd(q, k, v, do, lengths, causal, w, bucket):
    """Values in 64 bits from the definition; a query whose keys all have weight -inf meets none."""
    reach = bucket.numel() // 2
    leaves = [t.double().requires_grad_() for t in (q, k, v, w)]
    q64, k64, v64, w64 = leaves
    group, outs = q.shape[1] // k.shape[1], []
    for n, s in zip(lengths, _starts(lengths)):
        i = torch.arange(n, device=DEV)
        far = i[None] - i[:, None]
        z = q64[s:s + n].transpose(0, 1) @ k64[s:s + n].transpose(0, 1).repeat_interleave(group, 0).transpose(1, 2) * 0.125
        bias = w64[:, bucket.long()[far.clamp(-reach, reach) + reach]]
        seen = (bias != -math.inf) & (far <= 0 if causal else torch.ones_like(far, dtype=torch.bool))
        z = torch.where(seen, z + torch.where(seen, bias, 0.0), -1e300)
        p = torch.softmax(z, 2) * seen.any(2, keepdim=True)
        outs.append((p @ v64[s:s + n].transpose(0, 1).repeat_interleave(group, 0)).transpose(0, 1))
    out = torch.cat(outs)
    out.backward(do.double())
    return dict(out=out.detach(), dq=q64.grad, dk=k64.grad, dv=v64.grad, dw=w64.grad)


@BOTH_TYPES
@BOTH_WAYS
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
@pytest.mark.parametrize("reach", [3, 128])
def test_weights_of_minus_infinity_hide_keys(lengths, reach, causal, dtype):
    """Head 0: no key at all; head 1: not a query's own key, so that a text's first query (causal) meets none; head 2:
    no key past reach.  The bounds are those of weights of -300, whose keys weigh nothing either."""
    q, k, v, do = _inputs(lengths, 4, 2, 64, dtype, 7)
    bucket = lram.relative_buckets(8, reach)
    w = torch.randn((4, 8), generator=torch.Generator().manual_seed(8)).to(DEV).to(dtype)
    w[0] = w[1, 0] = w[2, bucket[0]] = w[2, bucket[-1]] = -math.inf
    got = _run(q, k, v, do, lengths, causal, w, bucket)
    value = _by_autograd(q, k, v, do, lengths, causal, w, bucket)
    like = ref.attention(q, k, v, lengths, lengths, _starts(lengths), _starts(lengths), causal, 0.125,
                         w.clamp(min=-300.0), bucket, do)
    for n in value:
        ref.assert_close(n, got[n], (value[n], like[n][1]))
    assert not got["out"][:, 0].any() and not got["dq"][:, 0].any() and not got["dw"][0].any()
    assert (got["lse"][:, 0] == -math.inf).all()
    if causal:
        first = _starts(lengths)
        assert not got["out"][first, 1].any() and not got["dq"][first, 1].any()



def _with_bounds(q, k, v, do, lengths, causal, w, bucket):
    """{name: (value, bound)} where finite weights beyond 1e8 are vast: a key counts only if its weight is of the highest kind
    (+vast, ordinary, -vast) that its query meets, and beside a vast weight the score does not count.  The bounds are
    layer_reference.attention's; a vast row's z are exact, and its lse holds log2 of a count to 2^-18."""
    e, reach, dt, d, scale = ref.E, bucket.numel() // 2, q.dtype, q.shape[2], 0.125
    u, r, hk, group = ref.HALF[dt], ref.half_operand(dt), k.shape[1], q.shape[1] // k.shape[1]
    got = {n: [torch.zeros(t.shape, dtype=torch.float64, device=DEV) for _ in range(2)]
           for n, t in dict(out=q, dq=q, dk=k, dv=v, dw=w).items()}

    def put(name, at, value, bound):
        for t, x in zip(got[name], (value, bound)):
            t[at] = x.transpose(0, 1)

    def shared(t):
        return t.unflatten(0, (hk, group)).sum(1)

    for n, s in zip(lengths, _starts(lengths)):
        rows = slice(s, s + n)
        q64, g64 = (t[rows].double().transpose(0, 1) for t in (q, do))
        k64, v64 = (t[rows].double().transpose(0, 1).repeat_interleave(group, 0) for t in (k, v))
        i = torch.arange(n, device=DEV)
        far = i[None] - i[:, None]
        of = bucket.long()[far.clamp(-reach, reach) + reach]
        bias = w.double()[:, of]
        kind = torch.where(bias.abs() > 1e8, bias.sign(), 0.0)
        kind = kind.masked_fill(far > 0, -2.0) if causal else kind
        top = kind.amax(2, keepdim=True)
        score = q64 @ k64.transpose(1, 2) * scale
        z = torch.where(top == 0, score + bias, 0.0).masked_fill(kind != top, -math.inf)
        dz = (d + 8) * e * scale * (q64.abs() @ k64.abs().transpose(1, 2)) + 8 * e * (score.abs() + bias.abs())
        dz = torch.where(top == 0, dz.masked_fill(kind != top, 0.0), 44 * e)
        p = torch.softmax(z, 2)
        dp = 2 * (dz.amax(2, keepdim=True) + 16 * e)
        o = p @ v64
        raw = (r + dp + (n + 16) * e) * (p @ v64.abs())
        put("out", rows, o, (u + e) * o.abs() + raw)
        delta = (g64 * o).sum(2, keepdim=True)
        ddelta = ((g64.abs() * (raw + 2.0 ** -17 * o.abs())).sum(2, keepdim=True) +
                  (d + 8) * e * (g64 * o).abs().sum(2, keepdim=True))
        t = g64 @ v64.transpose(1, 2) - delta
        ds = p * t
        raw_ds = p * (dp * t.abs() + (d + 8) * e * (g64.abs() @ v64.abs().transpose(1, 2)) + ddelta) + 4 * e * ds.abs()
        dds, many = raw_ds + r * ds.abs(), (n * group + 16) * e
        dq = scale * (ds @ k64)
        put("dq", rows, dq, u * dq.abs() + scale * ((dds + (n + 8) * e * ds.abs()) @ k64.abs()))
        dk, dv = scale * shared(ds.transpose(1, 2) @ q64), shared(p.transpose(1, 2) @ g64)
        put("dk", rows, dk, u * dk.abs() + scale * shared((dds + many * ds.abs()).transpose(1, 2) @ q64.abs()))
        put("dv", rows, dv, u * dv.abs() + shared(((r + dp + many) * p).transpose(1, 2) @ g64.abs()))
        for c in range(w.shape[1]):
            got["dw"][0][:, c] += (ds * (of == c)).sum((1, 2))
            got["dw"][1][:, c] += ((raw_ds + (many + n * e) * ds.abs()) * (of == c)).sum((1, 2))
    got["dw"][1] += u * got["dw"][0].abs()
    return got


@BOTH_TYPES
@BOTH_WAYS
@pytest.mark.parametrize("lengths", LENGTHS + [[1200, 3]], ids=str)
@pytest.mark.parametrize("reach", [3, 128])
def test_vast_weights(lengths, reach, causal, dtype):
    """Head 0: every weight the type's lowest value; head 1: that for a query's own key; head 2: -1e9 everywhere; head 3:
    +1e9 for one bucket, the lowest value for a query's own key's and one past reach."""
    q, k, v, do = _inputs(lengths, 4, 2, 64, dtype, 10)
    bucket = lram.relative_buckets(8, reach)
    w = torch.randn((4, 8), generator=torch.Generator().manual_seed(9)).to(DEV).to(dtype)
    w[0] = w[1, 0] = w[3, 0] = w[3, bucket[-1]] = torch.finfo(dtype).min
    w[2], w[3, bucket[reach - 1]] = -1e9, 1e9
    got = _run(q, k, v, do, lengths, causal, w, bucket)
    want = _with_bounds(q, k, v, do, lengths, causal, w, bucket)
    for n in want:
        ref.assert_close(n, got[n], want[n])


def test_the_form_with_vast_weights_is_the_other_one_without():
    lengths = [33, 70]
    q, k, v, do = _inputs(lengths, 4, 2, 64, F32, 12)
    w, bucket = torch.randn((4, 8), device=DEV), lram.relative_buckets(8, 20)
    got = _with_bounds(q, k, v, do, lengths, True, w, bucket)
    want = ref.attention(q, k, v, lengths, lengths, _starts(lengths), _starts(lengths), True, 0.125, w, bucket, do)
    for n, t in got.items():
        assert torch.allclose(t[0], want[n][0], rtol=1e-12, atol=1e-12), n
        assert torch.allclose(t[1], want[n][1], rtol=1e-3, atol=1e-12), n


@BOTH_TYPES
@pytest.mark.parametrize("nq,nk", [([1, 1], [5000, 70]), ([70], [4111]), ([40, 100], [300, 3000])], ids=str)
def test_vast_weights_over_a_cache(nq, nk, dtype):
    """Divided keys, whose pieces are joined by their lse: where every weight is the lowest value, out is the mean of the
    values, as with scores that are all 0."""
    g = torch.Generator(device=DEV)
    g.manual_seed(11)
    k, v = (torch.randn((sum(nk), 2, 64), generator=g, device=DEV).to(dtype) for _ in range(2))
    q, do = (torch.randn((sum(nq), 4, 64), generator=g, device=DEV).to(dtype) for _ in range(2))
    rel = lram.RelativeBias(torch.full((4, 8), torch.finfo(dtype).min, dtype=dtype, device=DEV), lram.relative_buckets(8, 30))
    seqs = lram.pack(nq, nk)
    out, saved = lram.attention_forward(q, k, v, seqs, rel=rel, save=True)
    dq, dk, dv, dw = lram.attention_backward(q, k, v, seqs, out, saved, do, rel=rel)
    zero = ref.attention(q * 0, k, v, nq, nk, _starts(nq), _starts(nk), False, 0.125, do=do)
    # p has one term more than there: what is left of log2 of the count, 2^-18
    more = {"out": 2 * 44 * ref.E * ref.attention(q * 0, k, v.abs(), nq, nk, _starts(nq), _starts(nk), False, 0.125)["out"][0]}
    ref.assert_close("out", out, (zero["out"][0], zero["out"][1] + more["out"]))
    ref.assert_close("dv", dv, (zero["dv"][0], zero["dv"][1] + 2 * 44 * ref.E * ref.attention(
        q * 0, k, v, nq, nk, _starts(nq), _starts(nk), False, 0.125, do=do.abs())["dv"][0]))


@BOTH_TYPES
@BOTH_WAYS
def test_vast_weights_beside_scores_of_next_to_nothing(causal, dtype):
    """A scale that makes every score 0: the mean of the values that are seen, in blocks with keys that are not, too."""
    lengths = [33, 150]
    q, k, v, do = _inputs(lengths, 4, 2, 64, dtype, 15)
    w = torch.full((4, 8), torch.finfo(dtype).min, dtype=dtype, device=DEV)
    rel, seqs = lram.RelativeBias(w, lram.relative_buckets(8, 3)), lram.pack(lengths)
    out, saved = lram.attention_forward(q, k, v, seqs, causal, 1e-20, rel, save=True)
    dq, dk, dv, dw = lram.attention_backward(q, k, v, seqs, out, saved, do, causal, 1e-20, rel)
    want = _with_bounds(q, k, v, do, lengths, causal, w, rel.bucket)
    for n, t in dict(out=out, dv=dv).items():
        ref.assert_close(n, t, want[n])
    assert all(torch.isfinite(t).all() for t in (dq, dk, dw))


@BOTH_TYPES
@pytest.mark.parametrize("nq,nk", [([1, 5], [20, 33]), ([40, 1], [45, 70]), ([130], [150])], ids=str)
@pytest.mark.parametrize("reach", [2, 10])
def test_weights_that_no_pair_meets(nq, nk, reach, dtype):
    """Buckets of keys behind the query, in causal attention: whatever their weights hold, NaN among it, nothing changes."""
    g = torch.Generator(device=DEV)
    g.manual_seed(13)
    q, do = (torch.randn((sum(nq), 4, 64), generator=g, device=DEV).to(dtype) for _ in range(2))
    k, v = (torch.randn((sum(nk), 4, 64), generator=g, device=DEV).to(dtype) for _ in range(2))
    bucket, seqs = lram.relative_buckets(8, reach), lram.pack(nq, nk)
    got = []
    for unmet in (0.0, math.nan, math.inf, -math.inf):
        w = torch.randn((4, 8), generator=torch.Generator().manual_seed(14)).to(DEV).to(dtype)
        w[:, 4:] = unmet
        rel = lram.RelativeBias(w, bucket)
        out, saved = lram.attention_forward(q, k, v, seqs, True, rel=rel, save=True)
        got.append((out, saved.lse, *lram.attention_backward(q, k, v, seqs, out, saved, do, True, rel=rel)))
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))
