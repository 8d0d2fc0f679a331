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
