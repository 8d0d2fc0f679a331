"""Rotary positions against the rotation in 64 bits, with bounds from the arithmetic that the header states."""
import pytest
import torch
from torch.autograd import forward_ad

import cache_reference as ref
import paper_2107_03474_amd as lram

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def _randn(g, *shape, dtype=F32):
    return torch.randn(shape, generator=g, device=DEV).to(dtype)


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


CASES = [
    # rows, heads, kv_heads, head_dim, pairs, interleaved, first position, dtype
    (1, 8, 8, 64, 32, False, 777, BF16),
    (37, 8, 2, 64, 32, True, 0, BF16),
    (130, 4, 4, 128, 64, False, 1 << 20, F32),
    (9, 12, 4, 64, 17, False, 1000003, F32),
    (9, 12, 4, 64, 17, True, 1000003, BF16),
    (5, 3, 1, 40, 1, False, (1 << 31) - 6, BF16),
    (5, 3, 1, 40, 1, True, -(1 << 31), F32),
    (3, 1, 1, 8, 4, False, -5, BF16),
    (3, 2, 0, 8, 3, True, -5, F32),
    (2, 5, 3, 1024, 512, False, 123456789, BF16),
    (700, 16, 8, 128, 32, False, 5000, BF16),
    (4100, 24, 4, 96, 48, False, 100, BF16),
    (4100, 24, 4, 96, 45, True, 100, F32),
]


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("rows,heads,kv,dim,pairs,interleaved,first,dtype", CASES)
def test_values(rows, heads, kv, dim, pairs, interleaved, first, dtype, backward):
    g = _gen(rows + pairs)
    x = _randn(g, rows, (heads + kv) * dim + 16, dtype=dtype)  # slices of wider rows
    q = x[:, :heads * dim].unflatten(1, (heads, dim))
    k = x[:, heads * dim:(heads + kv) * dim].unflatten(1, (kv, dim)) if kv else None
    at = (torch.arange(rows, device=DEV) + first).to(torch.int32)
    plan = lram.rotary_plan(2 * pairs, interleaved=interleaved)._replace(magnitude=1.25)
    call = lram.rotary_backward if backward else lram.rotary_forward
    got = call(q, k, at, plan)
    again = call(q, k, at, plan)
    for y, z, x1 in zip(got, again, (q, k)):
        if x1 is None:
            assert y is None
            continue
        assert y.is_contiguous() and y.dtype == dtype and torch.equal(y, z)
        ref.check(y, ref.rotated(x1, at, plan.turns, interleaved, 1.25, backward))
        assert torch.equal(y[..., 2 * pairs:], x1[..., 2 * pairs:])


def test_heads_before_rows():
    """[heads, rows, D] tensors."""
    g = _gen(1)
    x = _randn(g, 6, 50, 64, dtype=BF16)
    at = torch.randint(-(1 << 31), (1 << 31) - 1, (50,), generator=g, device=DEV).to(torch.int32)
    plan = lram.rotary_plan(64)
    got, _ = lram.rotary_forward(x.transpose(0, 1), None, at, plan)
    dense = x.transpose(0, 1).contiguous()
    want, _ = lram.rotary_forward(dense, None, at, plan)
    assert torch.equal(got, want)


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradients(interleaved):
    """Autograd's gradients are the rotation back, and the differences of a linear map."""
    g = _gen(2)
    q, k = (_randn(g, 11, h, 32).requires_grad_() for h in (4, 2))
    at = torch.randint(0, 100000, (11,), generator=g, device=DEV).to(torch.int32)
    plan = lram.rotary_plan(24, interleaved=interleaved, scaling="parts", factor=4.0, length=512)
    a, b = lram.rotary(q, k, at, plan)
    ga, gb = _randn(g, 11, 4, 32), _randn(g, 11, 2, 32)
    torch.autograd.backward((a, b), (ga, gb))
    ref.check(q.grad, ref.rotated(ga, at, plan.turns, interleaved, plan.magnitude, True))
    ref.check(k.grad, ref.rotated(gb, at, plan.turns, interleaved, plan.magnitude, True))
    d = _randn(g, 11, 4, 32)
    with torch.no_grad():
        step = lram.rotary(q + 0.5 * d, None, at, plan)[0].double() - lram.rotary(q - 0.5 * d, None, at, plan)[0].double()
    assert abs(float((step * ga).sum() - (d.double() * q.grad).sum())) < 1e-3  # 1,408 terms of rounding 2^-23 at most 4 each
    for only in (0, 1):  # one of the two is used
        q.grad = k.grad = None
        y = lram.rotary(q, k, at, plan)[only]
        y.backward((ga, gb)[only].transpose(0, 1).contiguous().transpose(0, 1))  # a gradient of other strides
        assert (q.grad is None) == bool(only) and (k.grad is None) == (not only)
        ref.check((k if only else q).grad, ref.rotated((gb if only else ga), at, plan.turns, interleaved, plan.magnitude, True))
    for only in (0, 1):  # one of the two is trained
        x = [t.detach().requires_grad_(i == only) for i, t in enumerate((q, k))]
        torch.autograd.backward(lram.rotary(*x, at, plan), (ga, gb))
        assert x[1 - only].grad is None
        ref.check(x[only].grad, ref.rotated((ga, gb)[only], at, plan.turns, interleaved, plan.magnitude, True))
    x = _randn(g, 11, 1, 32).requires_grad_()  # a gradient that is broadcast, of an odd start
    lram.rotary(x, None, at, plan)[0].sum().backward()
    ref.check(x.grad, ref.rotated(torch.ones_like(x), at, plan.turns, interleaved, plan.magnitude, True))


def test_second_derivatives_are_refused():
    g = _gen(3)
    q = _randn(g, 3, 2, 16).requires_grad_()
    at = torch.arange(3, dtype=torch.int32, device=DEV)
    y, _ = lram.rotary(q, None, at, lram.rotary_plan(16))
    first, = torch.autograd.grad((y * y).sum(), q, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(first.sum(), q)


def test_forward_mode_is_refused():
    q = torch.randn((3, 2, 16), device=DEV)
    at, plan = torch.arange(3, dtype=torch.int32, device=DEV), lram.rotary_plan(16)
    with forward_ad.dual_level():
        with pytest.raises(NotImplementedError):
            lram.rotary(forward_ad.make_dual(q, torch.ones_like(q)), None, at, plan)
        lram.rotary(q, None, at, plan)  # no tangent: nothing to refuse


@pytest.mark.parametrize("interleaved,pairs,dtype", [(False, 32, BF16), (True, 30, BF16), (False, 13, F32)])
def test_many_rows_are_rotated_as_few(interleaved, pairs, dtype):
    """Results past the caches, and threads that go over several heads: the bits of the same rows by themselves."""
    g = _gen(5)
    rows = 18000 if dtype == BF16 else 9000
    q, k = _randn(g, rows, 12, 64, dtype=dtype), _randn(g, rows, 5, 64, dtype=dtype)
    at = torch.randint(-(1 << 31), (1 << 31) - 1, (rows,), generator=g, device=DEV).to(torch.int32)
    plan = lram.rotary_plan(2 * pairs, interleaved=interleaved)
    a, b = lram.rotary_forward(q, k, at, plan)
    assert a.numel() * a.element_size() + b.numel() * b.element_size() > 32 << 20
    for first in (0, 777, rows - 40):
        part = slice(first, first + 40)
        x, y = lram.rotary_forward(q[part], k[part], at[part], plan)
        assert torch.equal(a[part], x) and torch.equal(b[part], y)


@pytest.mark.parametrize("lengths,before,after", [([5, 0, 17, 1], 2, 3), ([1] * 300, 0, 0), ([0], 3, 0), ([], 0, 4)])
def test_positions(lengths, before, after):
    seqs = lram.pack(lengths)
    seqs = seqs._replace(start_q=seqs.start_q + before)
    rows = sum(lengths) + before + after
    first = [7 * b + 1 for b in range(len(lengths))]
    want = [0] * before + [f + i for f, n in zip(first, lengths) for i in range(n)] + [0] * after
    got = lram.packed_positions(seqs, rows, torch.tensor(first, dtype=torch.int32, device=DEV))
    assert got.tolist() == want
    assert lram.packed_positions(seqs, rows).tolist() == [0] * before + [i for n in lengths for i in range(n)] + [0] * after
    assert lram.packed_positions(seqs, 0).numel() == 0


def test_refusals():
    q = torch.zeros((4, 2, 64), device=DEV)
    at, plan = torch.zeros(4, dtype=torch.int32, device=DEV), lram.rotary_plan(64)
    for bad, what in ((dict(q=q[..., :60]), "multiple of 8"), (dict(q=torch.zeros((4, 2, 68), device=DEV)[..., 2:66]), "16 bytes"),
                      (dict(q=q[:1].expand(4, 2, 64)), "16 bytes"), (dict(q=q.double()), "float32 or bfloat16"),
                      (dict(q=q[0]), r"\[rows, heads"), (dict(at=at[:3]), "position"), (dict(at=at.long()), "position"),
                      (dict(k=q.bfloat16()), "q's device, type"), (dict(k=q[:3]), "same rows"), (dict(q=q[:, :0]), "have heads"),
                      (dict(plan=lram.rotary_plan(66)), "1 to head_dim / 2"), (dict(plan=plan._replace(turns=plan.turns[:0])), "1 to"),
                      (dict(plan=plan._replace(magnitude=float("nan"))), "magnitude"),
                      (dict(plan=plan._replace(turns=plan.turns.int())), "turns"), (dict(plan=lram.rotary_plan(64, device="cpu")), "GPU")):
        a = dict(dict(q=q, k=None, at=at, plan=plan), **bad)
        with pytest.raises(lram.LramError, match=what):
            lram.rotary_forward(a["q"], a["k"], a["at"], a["plan"])
    empty = lram.rotary_forward(q[:0], q[:0], at[:0], plan)
    assert empty[0].shape == empty[1].shape == (0, 2, 64)


def test_a_captured_call_and_a_side_stream():
    g = _gen(4)
    q, k = _randn(g, 20, 4, 64, dtype=BF16), _randn(g, 20, 2, 64, dtype=BF16)
    at = torch.arange(20, dtype=torch.int32, device=DEV)
    plan = lram.rotary_plan(64)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = lram.rotary_forward(q, k, at, plan)
    torch.cuda.current_stream().wait_stream(s)
    for a, b in zip(got, lram.rotary_forward(q, k, at, plan)):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = lram.rotary_forward(q, k, at, plan)
    for i in range(4):
        q.copy_(_randn(g, 20, 4, 64, dtype=BF16))
        at.add_(1000 * i)
        want = lram.rotary_forward(q, k, at, plan)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


def test_a_captured_training_step():
    """Forward and backward in one graph, of leaves that no other graph holds, over other values at every replay."""
    g = _gen(5)
    q, k = (_randn(g, 37, h, 64, dtype=BF16).requires_grad_() for h in (4, 2))
    gq, gk = _randn(g, 37, 4, 64, dtype=BF16), _randn(g, 37, 2, 64, dtype=BF16)
    at = torch.arange(37, dtype=torch.int32, device=DEV)
    plan = lram.rotary_plan(48, interleaved=True)

    def step():
        a, b = lram.rotary(q, k, at, plan)
        return (a.detach(), b.detach(), *torch.autograd.grad((a, b), (q, k), (gq, gk)))

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(2):
            step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for i in range(4):
        with torch.no_grad():
            q.copy_(_randn(g, 37, 4, 64, dtype=BF16))
            gk.copy_(_randn(g, 37, 2, 64, dtype=BF16))
            at.add_(77 * i)
        eager = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, eager))
