"""Packed attention whose first sequence does not start at row 0: some users of a shared cache, a batch inside a larger
buffer.  Against the 64-bit form and its derived bounds (layer_reference.py)."""
import pytest
import torch

import layer_reference as ref
import paper_2107_03474_amd as lram

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


def _randn(g, shape, dtype):
    return torch.randn(shape, generator=g, device=DEV).to(dtype)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("nq", [[1, 1], [5, 70]], ids=str)
def test_some_users_of_a_shared_cache(nq, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    cap, nk = 300, [70, 251]
    start = torch.arange(7, dtype=torch.int32, device=DEV) * cap
    k, v = (_randn(g, (6 * cap, 2, 64), dtype) for _ in range(2))
    q = _randn(g, (sum(nq), 4, 64), dtype)
    seqs = lram.Packed(_i32([0, nq[0], sum(nq)]), start[3:6], max(nq), max(nk), _i32(nk))  # users 3 and 4
    out, _ = lram.attention_forward(q, k, v, seqs, True)
    want = ref.attention(q, k, v, nq, nk, [0, nq[0]], [3 * cap, 4 * cap], True, 0.125)
    ref.assert_close("out", out, want["out"])


def _inside(lengths, front_q, front_k, behind, hq, hk, d, dtype, rel):
    """A batch with rows in front of it and behind it that belong to no sequence: zeros everywhere."""
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    n = sum(lengths)
    q, do = (_randn(g, (front_q + n + behind, hq, d), dtype) for _ in range(2))
    k, v = (_randn(g, (front_k + n + behind, hk, d), dtype) for _ in range(2))
    at = [sum(lengths[:i]) for i in range(len(lengths) + 1)]
    seqs = lram.Packed(_i32([front_q + a for a in at]), _i32([front_k + a for a in at]), max(lengths, default=0),
                       max(lengths, default=0))
    bias = lram.RelativeBias(_randn(g, (hq, 8), dtype), lram.relative_buckets(8, 20)) if rel else None
    out, saved = lram.attention_forward(q, k, v, seqs, True, rel=bias, save=True)
    dq, dk, dv, dw = lram.attention_backward(q, k, v, seqs, out, saved, do, True, rel=bias)
    torch.cuda.synchronize()
    want = ref.attention(q, k, v, lengths, lengths, [front_q + a for a in at[:-1]], [front_k + a for a in at[:-1]], True,
                         d ** -0.5, bias.weight if rel else None, bias.bucket if rel else None, do)
    got = dict(out=out, lse=saved.lse, dq=dq, dk=dk, dv=dv)
    if rel:
        got["dw"] = dw
    for name, t in got.items():
        ref.assert_close(name, t, want[name])
        if name in ("out", "dq", "dk", "dv"):
            front = front_k if name in ("dk", "dv") else front_q
            assert not t[:front].any() and not t[front + n:].any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("front_q,front_k,behind", [(1, 0, 0), (0, 1, 0), (200, 333, 50), (31, 700, 0)])
def test_a_batch_inside_larger_buffers(front_q, front_k, behind, dtype):
    for lengths in ([70], [300, 0, 41], [128, 128]):
        _inside(lengths, front_q, front_k, behind, 4, 2, 64, dtype, True)
        _inside(lengths, front_q, front_k, behind, 2, 2, 128, dtype, False)


def test_no_sequences_inside_buffers():
    _inside([], 70, 40, 33, 4, 2, 64, BF16, True)


@pytest.mark.parametrize("n", [61, 62, 63, 64, 200])
def test_many_sequences_inside_buffers(n):
    _inside([(37 * i) % 50 for i in range(n)], 130, 77, 9, 4, 2, 32, BF16, True)
    _inside([5] * n, 0, 1000, 0, 2, 1, 32, F32, False)
