"""Attention whose relative position bias has weights far from zero, against the 64-bit form and its derived bounds
(layer_reference.py)."""
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
