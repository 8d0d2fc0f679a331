"""Packed attention and its relative position bias on the GPU against the plain 64-bit form and its derived bounds
(layer_reference.py)."""
import pytest
import torch

import layer_reference as ref
import paper_2107_03474_amd as lram

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


def _randn(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def _starts(n):
    return [sum(n[:i]) for i in range(len(n))]


def _case(nq, nk, hq, hk, d, dtype, causal, rel=None, train=True, capacity=0, scale=None, layout="fused", wtype=None,
          hints=None, seed=0, sharp=1.0):
    """Runs a case and checks every result; returns what was run.  rel: (buckets, reach, both)."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed + sum(nq) + 7 * sum(nk))
    tq, tk = sum(nq), capacity * len(nk) if capacity else sum(nk)
    if layout == "fused" and tq == tk:
        x = _randn(g, (tq, (hq + 2 * hk) * d), dtype)
        q, k, v = (x[:, a * d:b * d].unflatten(1, (b - a, d)) for a, b in ((0, hq), (hq, hq + hk), (hq + hk, hq + 2 * hk)))
    elif layout == "heads":  # [heads, rows, head_dim]
        q = _randn(g, (hq, tq, d), dtype).transpose(0, 1)
        k, v = (_randn(g, (hk, tk, d), dtype).transpose(0, 1) for _ in range(2))
    else:
        q = _randn(g, (tq, hq, d), dtype)
        k, v = (_randn(g, (tk, hk, d), dtype) for _ in range(2))
    if sharp != 1.0:
        q = q * sharp
    seqs = lram.pack(nq, nk, capacity)
    sk = [i * capacity for i in range(len(nk))] if capacity else _starts(nk)
    if capacity:  # what a cache holds past its sequence is never met
        for s, n in zip(sk, nk):
            k[s + n:s + capacity] = float("nan")
            v[s + n:s + capacity] = float("inf")
    if hints is not None:
        seqs = seqs._replace(max_q=hints[0], max_k=hints[1])
    bias = None
    if rel is not None:
        bucket = lram.relative_buckets(*rel) if isinstance(rel[0], int) else torch.tensor(rel[1], dtype=torch.int32, device=DEV)
        buckets = rel[0] if isinstance(rel[0], int) else max(rel[1]) + 1
        bias = lram.RelativeBias(_randn(g, (hq, buckets), wtype or dtype), bucket)
    do = _randn(g, (tq, hq, d), dtype)
    s = d ** -0.5 if scale is None else scale
    out, saved = lram.attention_forward(q, k, v, seqs, causal, scale, bias, save=train)
    got = {"out": out}
    if train:
        got["lse"] = saved.lse
        got["dq"], got["dk"], got["dv"], dw = lram.attention_backward(q, k, v, seqs, out, saved, do, causal, scale, bias)
        if bias is not None:
            got["dw"] = dw
    torch.cuda.synchronize()
    want = ref.attention(q, k, v, nq, nk, _starts(nq), sk, causal, s, None if bias is None else bias.weight,
                         None if bias is None else bias.bucket, do if train else None)
    for n, t in got.items():
        assert t.dtype == (F32 if n == "lse" else bias.weight.dtype if n == "dw" else dtype)
        ref.assert_close(n, t, want[n])
    return q, k, v, seqs, bias, do, got


LENGTHS = [[1], [2, 0, 1], [31, 32, 33], [63, 64, 65], [127, 128, 129, 5], [300, 1, 77]]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
def test_packed(lengths, causal, d, dtype):
    _case(lengths, lengths, 4, 2, d, dtype, causal)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("hq,hk", [(1, 1), (3, 1), (6, 2), (8, 1), (10, 2), (64, 1), (16, 16)])
def test_head_groups(hq, hk, dtype):
    _case([70, 3, 40], [70, 3, 40], hq, hk, 32, dtype, True)
    _case([1, 3, 9], [50, 64, 130], hq, hk, 64, dtype, True)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("nq,nk", [([5, 1, 40], [3, 0, 200]), ([130, 7], [64, 2]), ([200], [1]), ([1, 1], [0, 0]),
                                   ([33, 64], [97, 500])], ids=str)
@pytest.mark.parametrize("causal", [False, True])
def test_other_key_counts(nq, nk, causal, dtype):
    """Fewer keys than queries leave causal rows empty; no keys leave every row empty."""
    _case(nq, nk, 4, 2, 64, dtype, causal, rel=(16, 20, True))
    _case(nq, nk, 2, 1, 128, dtype, causal)


@pytest.mark.parametrize("dtype,wtype", [(F32, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("rel", [(32, 128, True), (8, 5, False), (2, 1, True), ("table", [0]), ("table", [3, 1, 0, 2, 7])],
                         ids=str)
@pytest.mark.parametrize("causal", [False, True])
def test_bias(rel, causal, dtype, wtype):
    _case([200, 1, 65], [200, 1, 65], 4, 2, 64, dtype, causal, rel=rel, wtype=wtype)
    _case([450], [450], 1, 1, 128, dtype, causal, rel=rel, wtype=wtype)
    _case([1, 2, 4], [333, 65, 4], 6, 2, 32, dtype, causal, rel=rel, wtype=wtype, capacity=400)


def test_bias_of_a_large_group_and_reach():
    _case([90, 10], [90, 10], 8, 1, 64, BF16, True, rel=(32, 128, True))
    _case([300], [300], 1, 1, 32, F32, False, rel=(64, 1900, True))
    _case([3], [300], 8, 1, 64, BF16, True, rel=(32, 128, False))


@pytest.mark.parametrize("d,dtype,reach", [(128, BF16, 1951), (128, F32, 586), (64, F32, 1951), (128, BF16, 313),
                                           (128, BF16, 314)])
def test_the_longest_reach(d, dtype, reach):
    _case([500], [500], 2, 2, d, dtype, True, rel=(64, reach, True))


@pytest.mark.parametrize("layout", ["heads", "separate"])
def test_layouts(layout):
    _case([90, 33], [90, 33], 4, 2, 64, BF16, True, layout=layout)
    _case([2, 33], [90, 33], 4, 2, 32, F32, True, layout=layout, rel=(8, 8, True))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_tokens_over_a_cache(d, dtype):
    for bias in (None, (32, 128, True)):
        _case([1] * 5, [1, 31, 128, 129, 700], 8, 2, d, dtype, True, train=False, capacity=701, rel=bias)
        _case([4, 1, 3], [4, 900, 333], 4, 4, d, dtype, True, train=False, capacity=1000, rel=bias)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_divided_keys(dtype):
    """Few rows over many keys: pieces of the keys, joined; sequences with fewer keys than pieces."""
    for train in (False, True):
        _case([1, 1], [5000, 70], 4, 2, 64, dtype, True, train=train, layout="separate")
        _case([3, 2], [2100, 0], 2, 2, 32, dtype, False, train=train, layout="separate", rel=(16, 64, True))
    _case([100, 130], [6000, 1100], 2, 1, 128, dtype, True, layout="separate")
    _case([70], [4111], 1, 1, 64, dtype, True, layout="separate", rel=(32, 128, True))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_divided_rows(d, dtype):
    """Few key tiles under many rows: pieces of the rows, joined."""
    _case([1200, 3], [1200, 3], 4, 2, d, dtype, True)
    _case([2500], [130], 1, 1, d, dtype, False, layout="separate", rel=(16, 30, True))


def test_long_texts_among_short_ones():
    """Tiles enough for the chip, of sequences that differ much."""
    lengths = [2200, 3, 700, 0, 1100, 64]
    _case(lengths, lengths, 12, 12, 64, BF16, True, rel=(32, 128, True))
    _case(lengths, lengths, 16, 8, 128, BF16, False)


@pytest.mark.parametrize("group", [2, 5, 6, 8])
def test_rows_divided_by_heads(group):
    """Few queries of many heads on a key head: pieces of the rows are sets of heads."""
    for n in ([200], [64, 65], [300, 310, 290], [1]):
        _case(n, n, group, 1, 64, F32, True, rel=(16, 40, True))
        _case(n, n, 2 * group, 2, 32, F32, False)
    _case([5], [700], group, 1, 128, F32, True, layout="separate")
    _case([130], [70], group, 1, 128, BF16, False, layout="separate")


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_few_tiles_of_long_rows(causal, d):
    """Tiles of keys shared out among the waves of a workgroup: odd and even numbers of them, ends inside them."""
    for n in (257, 300, 384, 449, 1030, 1100):
        _case([n], [n], 4, 2, d, BF16, causal, rel=(32, 128, True) if n % 2 else None)
    _case([400, 390], [470, 130], 2, 2, d, BF16, causal, layout="separate")
    _case([600], [2500], 2, 1, d, BF16, causal, train=False, layout="separate", rel=(16, 64, True))


def test_hints_do_not_change_results():
    lengths = [150, 1, 290]
    for hints in ((0, 0), (1, 1), (1, 290), (290, 1), (10 ** 9, 10 ** 9), ((1 << 63) - 1,) * 2):
        _case(lengths, lengths, 4, 2, 64, BF16, True, hints=hints, rel=(32, 128, True))
        _case(lengths, lengths, 2, 1, 128, BF16, False, hints=hints)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_sharp_softmax(dtype):
    """Scores far apart: the running maximum moves often, weights underflow."""
    _case([260, 40], [260, 40], 4, 2, 64, dtype, True, sharp=12.0)
    _case([1], [3000], 2, 2, 64, dtype, True, train=False, sharp=12.0, layout="separate")


def test_scale():
    _case([100], [100], 2, 1, 64, BF16, True, scale=0.01)
    _case([100], [100], 2, 1, 64, F32, False, scale=1.7)


def test_rows_past_the_last_sequence_and_empty_batches():
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    q, k, v, do = (_randn(g, (50, 2, 64), BF16) for _ in range(4))
    seqs = lram.pack([20, 10])  # rows 30 ... 49 belong to no sequence
    out, saved = lram.attention_forward(q, k, v, seqs, save=True)
    dq, dk, dv, _ = lram.attention_backward(q, k, v, seqs, out, saved, do)
    want = ref.attention(q[:30], k[:30], v[:30], [20, 10], [20, 10], [0, 20], [0, 20], False, 0.125, do=do[:30])
    for n, t in (("out", out), ("dq", dq), ("dk", dk), ("dv", dv)):
        ref.assert_close(n, t[:30], want[n])
        assert not t[30:].any()
    assert (saved.lse[30:] == -float("inf")).all()
    none = lram.pack([])
    out, saved = lram.attention_forward(q, k, v, none, save=True)
    grads = lram.attention_backward(q, k, v, none, out, saved, do)
    assert not out.any() and not any(t.any() for t in grads[:3])
    e = q[:0]
    out, saved = lram.attention_forward(e, e, e, none, save=True)
    assert out.shape == (0, 2, 64)
    rel = lram.RelativeBias(torch.ones((2, 32), dtype=BF16, device=DEV), lram.relative_buckets(32, 128))
    grads = lram.attention_backward(e, e, e, none, out, saved, e, rel=rel)
    assert grads[0].shape == (0, 2, 64) and not grads[3].any()


def test_whatever_the_starts_hold_stays_inside():
    """Starts that do not ascend or pass the tensors: results mean nothing, and nothing outside is addressed."""
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    q, k, v, do = (_randn(g, (300, 2, 64), BF16) for _ in range(4))
    for sq, sk, used in (([0, 200, 100, 300], [0, 300, 10, 20], None), ([5, 400, -7, 1 << 30], [-5, 1 << 30, 7, 9], None),
                         ([0, 100, 200, 300], [0, 100, 200, 300], [1 << 30, -4, 50])):
        t = [torch.tensor(x, dtype=torch.int32, device=DEV) if x is not None else None for x in (sq, sk, used)]
        seqs = lram.Packed(t[0], t[1], 100, 100, t[2])
        rel = lram.RelativeBias(torch.ones((2, 4), dtype=BF16, device=DEV),
                                torch.tensor([-9, 1 << 30, 2, 77, 1], dtype=torch.int32, device=DEV))
        out, saved = lram.attention_forward(q, k, v, seqs, True, rel=rel, save=True)
        lram.attention_backward(q, k, v, seqs, out, saved, do, True, rel=rel)
        torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [62, 63, 64, 65, 300])
def test_many_sequences(n, dtype):
    """A lane to a sequence below 64, a search from there on; empty ones among them, first and last."""
    lengths = [(37 * i) % 150 if i % 5 and i < n - 2 else 0 for i in range(n)]
    _case(lengths, lengths, 4, 2, 32, dtype, True)
    lengths = [0 if i == 7 else 1 + (53 * i) % 40 for i in range(n)]
    _case(lengths, [1 + (29 * i) % 90 for i in range(n)], 2, 2, 64, dtype, True, rel=(8, 12, True))
    _case([1] * n, [(71 * i) % 130 for i in range(n)], 8, 2, 64, dtype, True, train=False, capacity=130)


def test_whatever_many_starts_hold_stays_inside():
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    q, k, v, do = (_randn(g, (300, 2, 64), BF16) for _ in range(4))
    rel = lram.RelativeBias(torch.ones((2, 4), dtype=BF16, device=DEV), torch.zeros(5, dtype=torch.int32, device=DEV))
    up = torch.arange(71, dtype=torch.int32, device=DEV) * 4
    for start in (up.flip(0).contiguous(), up * 1000, up - 140, (up * 37) % 301):
        seqs = lram.Packed(start, start, 100, 100, None)
        out, saved = lram.attention_forward(q, k, v, seqs, True, rel=rel, save=True)
        lram.attention_backward(q, k, v, seqs, out, saved, do, True, rel=rel)
        torch.cuda.synchronize()


def test_a_sequence_that_is_not_finite_stays_alone():
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    lengths = [40, 30, 70]
    q, k, v, do = (_randn(g, (140, 4, 64), BF16) for _ in range(4))
    v[45] = float("nan")
    k[50] = float("inf")
    seqs = lram.pack(lengths)
    out, saved = lram.attention_forward(q, k, v, seqs, True, save=True)
    dq, dk, dv, _ = lram.attention_backward(q, k, v, seqs, out, saved, do, True)
    for rows, n in ((slice(0, 40), 40), (slice(70, 140), 70)):
        want = ref.attention(q[rows], k[rows], v[rows], [n], [n], [0], [0], True, 0.125, do=do[rows])
        for name, t in (("out", out), ("dq", dq), ("dk", dk), ("dv", dv)):
            ref.assert_close(name, t[rows], want[name])
    assert torch.isnan(out[69].float()).all()


def test_a_cache_past_32_bits():
    """Keys and values of 5 GB: the last sequence's offsets pass 2^32 bytes and, in elements, 2^31."""
    cap, hk, d = 2_500_000 // 3, 8, 128
    k = torch.zeros((3 * cap, hk, d), dtype=BF16, device=DEV)
    v = torch.zeros_like(k)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    nq, nk = [1, 2, 70], [50, 3000, 900]
    for s, n in enumerate(nk):
        k[s * cap:s * cap + n] = _randn(g, (n, hk, d), BF16)
        v[s * cap:s * cap + n] = _randn(g, (n, hk, d), BF16)
    q = _randn(g, (sum(nq), 16, d), BF16)
    seqs = lram.pack(nq, nk, cap)
    out, _ = lram.attention_forward(q, k, v, seqs, True)
    want = ref.attention(q, k, v, nq, nk, _starts(nq), [0, cap, 2 * cap], True, d ** -0.5)
    ref.assert_close("out", out, want["out"])
    # one sequence that is that long itself: the last queries over its last keys (all others weigh nothing)
    n = 2_200_000
    k[:n] = -4.0
    k[n - 500:n] = _randn(g, (500, hk, d), BF16)
    v[n - 500:n] = _randn(g, (500, hk, d), BF16)
    q = q[:2].abs() + 1.0
    one = lram.pack([2], [n], 3 * cap)
    out, _ = lram.attention_forward(q, k, v, one, True)
    seen = ref.attention(q, k[n - 500:n], v[n - 500:n], [2], [500], [0], [0], True, d ** -0.5)
    ref.assert_close("out", out, (seen["out"][0], seen["out"][1] * 2))


def test_autograd():
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    lengths = [60, 5, 100]
    x = _randn(g, (165, 4 * 64 + 2 * 2 * 64), F32).requires_grad_()
    w = _randn(g, (4, 16), F32).requires_grad_()
    do = _randn(g, (165, 4, 64), F32)
    q, k, v = x[:, :256].unflatten(1, (4, 64)), x[:, 256:384].unflatten(1, (2, 64)), x[:, 384:].unflatten(1, (2, 64))
    bucket = lram.relative_buckets(16, 40)
    out = lram.attention(q, k, v, lram.pack(lengths), True, rel=lram.RelativeBias(w, bucket))
    (out * do).sum().backward()
    want = ref.attention(q.detach(), k.detach(), v.detach(), lengths, lengths, _starts(lengths), _starts(lengths), True,
                         0.125, w.detach(), bucket, do)
    ref.assert_close("dx", x.grad, tuple(torch.cat([want[n][i].flatten(1) for n in ("dq", "dk", "dv")], 1) for i in (0, 1)))
    ref.assert_close("dw", w.grad, want["dw"])


def test_without_gradients():
    q, k, v, seqs, bias, do, got = _case([60, 5], [60, 5], 4, 2, 64, BF16, True, rel=(16, 40, True))
    rel = lram.RelativeBias(bias.weight.requires_grad_(), bias.bucket)
    with torch.no_grad():
        out = lram.attention(q, k, v, seqs, True, rel=rel)
    assert not out.requires_grad and torch.equal(out, got["out"])
    out = lram.attention(q, k, v, seqs, True, rel=rel)
    assert out.requires_grad and torch.equal(out, got["out"])


def test_gradients_by_differences():
    """Directional differences of the kernel's own forward, in fp32, against its gradients: the forward's bounded errors
    over the step, and the third-order term taken from the 64-bit form's differences at the same step."""
    lengths = [20, 37]
    q, k, v, seqs, bias, do, got = _case(lengths, lengths, 4, 2, 32, F32, True, rel=(8, 12, True), layout="separate")
    step, args = 2.0 ** -6, [q, k, v, bias.weight]

    def sides(k_, t, d):
        side, side64, slack = [], [], 0.0
        for s in (step, -step):
            a = list(args)
            a[k_] = t + s * d
            out, _ = lram.attention_forward(*a[:3], seqs, True, rel=lram.RelativeBias(a[3], bias.bucket))
            o64, bound = ref.attention(*a[:3], lengths, lengths, _starts(lengths), _starts(lengths), True, 32 ** -0.5, a[3],
                                       bias.bucket)["out"]
            side.append(float((out.double() * do.double()).sum()))
            side64.append(float((o64 * do.double()).sum()))
            slack += float((bound * do.double().abs()).sum())
        return side, side64, slack

    want = ref.attention(*args[:3], lengths, lengths, _starts(lengths), _starts(lengths), True, 32 ** -0.5, args[3],
                         bias.bucket, do)
    for i, name in enumerate(("dq", "dk", "dv", "dw")):
        d = torch.sign(torch.randn_like(args[i]))
        side, side64, slack = sides(i, args[i], d)
        along, along64 = float((got[name].double() * d.double()).sum()), float((want[name][0] * d.double()).sum())
        curved = (side64[0] - side64[1]) / (2 * step) - along64
        moved = float((2.0 ** -24 * (args[i].abs() + step).double() * want[name][0].abs()).sum()) / step
        assert abs((side[0] - side[1]) / (2 * step) - curved - along) <= slack / (2 * step) + moved + float(want[name][1].sum())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_same_bits_every_time_and_in_a_graph(dtype):
    """Twice the same bits; a captured call replayed over other values and other lengths."""
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    lengths = [[400, 30, 70], [100, 100, 300], [500, 0, 0], [1, 498, 1]]
    q, k, v, do = (_randn(g, (500, 4, 64), dtype) for _ in range(4))
    k, v = k[:, :2], v[:, 2:]
    seqs = lram.pack(lengths[0])
    seqs = seqs._replace(max_q=500, max_k=500)
    rel = lram.RelativeBias(_randn(g, (4, 32), dtype), lram.relative_buckets(32, 128))

    def step():
        out, saved = lram.attention_forward(q, k, v, seqs, True, rel=rel, save=True)
        return (out, *lram.attention_backward(q, k, v, seqs, out, saved, do, True, rel=rel))

    step()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for n in lengths:
        other = lram.pack(n)
        seqs.start_q.copy_(other.start_q)
        seqs.start_k.copy_(other.start_k)
        q.copy_(_randn(g, q.shape, dtype))
        eager = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, captured))
        assert all(torch.equal(a, b) for a, b in zip(eager, step()))


def test_side_stream():
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    q, k, v, do = (_randn(g, (300, 4, 64), BF16) for _ in range(4))
    seqs = lram.pack([200, 100])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        big = torch.randn((4096, 4096), device=DEV)
        for _ in range(4):
            big = big @ big * 1e-3            # work in front of the call on the same stream
        q2 = q + 0 * big[:300, :256].view(300, 4, 64).nan_to_num(0, 0, 0).to(BF16)
        out, saved = lram.attention_forward(q2, k, v, seqs, save=True)
        grads = lram.attention_backward(q2, k, v, seqs, out, saved, do)
    s.synchronize()
    out2, saved2 = lram.attention_forward(q, k, v, seqs, save=True)
    grads2 = lram.attention_backward(q, k, v, seqs, out2, saved2, do)
    assert torch.equal(out, out2) and all(torch.equal(a, b) for a, b in zip(grads[:3], grads2[:3]))


def test_refuses():
    q = torch.zeros((8, 4, 64), dtype=BF16, device=DEV)
    k = torch.zeros((8, 2, 64), dtype=BF16, device=DEV)
    seqs = lram.pack([8])
    w, bucket = torch.zeros((4, 3), dtype=BF16, device=DEV), torch.zeros(5, dtype=torch.int32, device=DEV)
    ok = dict(q=q, k=k, v=k, seqs=seqs)
    lram.attention_forward(**ok)
    wide = torch.zeros((8, 4, 72), dtype=BF16, device=DEV)
    for bad in (dict(q=q[0]), dict(q=q.half()), dict(k=k.float()), dict(v=k[:, :1]), dict(v=k[:7]), dict(q=q.cpu()),
                dict(k=k.cpu()), dict(q=q[:, :3]), dict(q=q[..., :48], k=k[..., :48], v=k[..., :48]),
                dict(q=q.transpose(1, 2)), dict(q=wide[..., 4:68]), dict(q=q.expand(8, 4, 64)[:1].expand(8, 4, 64)),
                dict(seqs=seqs._replace(start_q=seqs.start_q.long())), dict(seqs=seqs._replace(start_k=seqs.start_k[:1])),
                dict(seqs=seqs._replace(used_k=seqs.start_k)), dict(seqs=seqs._replace(start_q=seqs.start_q.cpu())),
                dict(scale=0.0), dict(scale=float("nan")), dict(rel=lram.RelativeBias(w[:2], bucket)),
                dict(rel=lram.RelativeBias(w.half(), bucket)), dict(rel=lram.RelativeBias(w, bucket[:4])),
                dict(rel=lram.RelativeBias(w, bucket.long())), dict(rel=lram.RelativeBias(w.t(), bucket)),
                dict(rel=lram.RelativeBias(w, torch.zeros(2 * 2000 + 1, dtype=torch.int32, device=DEV)))):
        with pytest.raises(lram.LramError):
            lram.attention_forward(**dict(ok, **bad))
    out, saved = lram.attention_forward(**ok, save=True)
    for bad in (dict(out=out[:4]), dict(grad_out=out.float()), dict(saved=saved._replace(lse=saved.lse[:2])),
                dict(saved=saved._replace(residue=saved.residue.float()))):
        with pytest.raises(lram.LramError):
            lram.attention_backward(**dict(dict(ok, out=out, saved=saved, grad_out=out), **bad))
    with pytest.raises(lram.LramError, match="workspace"):
        lram.attention_backward(**ok, out=out, saved=saved, grad_out=out, workspace=torch.empty(16, device=DEV))
