"""Host-side checks of the layer's operators: exports, argument checks of the C ABI (nothing is launched), the bucket
table and the plans.  No GPU is needed."""
import ctypes
import math
import os
import re
import subprocess

import pytest
import torch

import layer_reference as ref
import paper_2107_03474_amd as lram
from paper_2107_03474_amd import layer

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000      # never dereferenced: every call here ends in the host's checks
EINVAL, EDTYPE, EWORKSPACE = 1, 3, 4


@pytest.fixture(scope="module")
def lib():
    return layer._library()


def test_every_declared_symbol_is_exported(lib):
    txt = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "lram_layer.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(lram_[a-z_0-9]+)\s*\(", txt))
    assert len(names) == 8
    out = subprocess.run(["nm", "-D", "--defined-only", lram.library_path()], capture_output=True, text=True,
                         check=True).stdout
    assert names <= set(re.findall(r"\bT (lram_[a-z_0-9]+)", out))


def _norm_fwd(lib, x=P, r=None, w=P, b=P, dt=1, wt=1, rows=4, width=64, eps=1e-5, h=None, y=P + 0x1000, mean=None,
              rstd=None):
    return lib.lram_layer_norm_forward(x, r, w, b, dt, wt, rows, width, eps, h, y, mean, rstd, None)


def _norm_bwd(lib, h=P, w=P, mean=P, rstd=P, dy=P, dh=None, dt=1, wt=1, rows=4000, width=64, dx=P, dw=P, db=P, ws=P,
              ws_bytes=1 << 30):
    return lib.lram_layer_norm_backward(h, w, mean, rstd, dy, dh, dt, wt, rows, width, dx, dw, db, ws, ws_bytes, None)


def test_norm_refuses(lib):
    for bad in (dict(x=None), dict(w=None), dict(b=None), dict(y=None), dict(x=P + 2), dict(y=P + 8), dict(w=P + 1),
                dict(rows=-1), dict(width=0), dict(width=16385), dict(eps=-1.0), dict(eps=math.nan), dict(r=P),
                dict(h=P), dict(mean=P), dict(rstd=P), dict(mean=P + 2, rstd=P), dict(r=P, h=P + 0x1000),
                dict(rows=1 << 31)):
        assert _norm_fwd(lib, **bad) == EINVAL, bad
    for bad in (dict(dt=2), dict(wt=2), dict(dt=0, wt=1)):
        assert _norm_fwd(lib, **bad) == EDTYPE, bad
    assert _norm_fwd(lib, rows=0, x=None, y=None) == 0
    for bad in (dict(h=None), dict(w=None), dict(mean=None), dict(rstd=None), dict(dy=None), dict(dx=None),
                dict(dw=None), dict(db=None), dict(dh=P + 4), dict(mean=P + 2), dict(db=P + 1), dict(width=0)):
        assert _norm_bwd(lib, **bad) == EINVAL, bad
    assert _norm_bwd(lib, dt=0, wt=1) == EDTYPE
    n = ctypes.c_size_t(0)
    assert lib.lram_layer_norm_backward_workspace_bytes(4000, 64, 1, ctypes.byref(n)) == 0 and n.value > 0
    for bad in (dict(ws=None), dict(ws=P + 4), dict(ws_bytes=n.value - 1)):
        assert _norm_bwd(lib, **bad) == EWORKSPACE, bad
    assert lib.lram_layer_norm_backward_workspace_bytes(1, 64, 1, ctypes.byref(n)) == 0 and n.value == 0
    assert lib.lram_layer_norm_backward_workspace_bytes(1, 64, 1, None) == EINVAL


def _describe(**kw):
    a = layer._Attention(dtype=1, wdtype=1, heads=8, kv_heads=4, head_dim=64, batch=2, causal=1, scale=0.125, tq=300,
                         tk=300, max_q=150, max_k=150, q=P, k=P, v=P, q_row=512, q_head=64, k_row=256, k_head=64,
                         v_row=256, v_head=64, start_q=P, start_k=P)
    for n, v in kw.items():
        setattr(a, n, v)
    return a


def _attention_fwd(lib, out=P, lse=P, residue=None, ws=P, ws_bytes=1 << 40, **kw):
    return lib.lram_attention_forward(ctypes.byref(_describe(**kw)), out, lse, residue, ws, ws_bytes, None)


def _attention_bwd(lib, out=P, residue=None, lse=P, do=P, dq=P, dk=P, dv=P, dw=None, ws=P, ws_bytes=1 << 40, **kw):
    return lib.lram_attention_backward(ctypes.byref(_describe(**kw)), out, residue, lse, do, dq, dk, dv, dw, ws,
                                       ws_bytes, None)


BIAS = dict(rel_weight=P, rel_bucket=P, rel_buckets=32, rel_reach=128)


def test_attention_refuses(lib):
    shared = [dict(heads=0), dict(kv_heads=0), dict(heads=6), dict(heads=65 * 4, kv_heads=4), dict(batch=-1),
              dict(causal=2), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan), dict(tq=-1),
              dict(tk=-1), dict(tk=1 << 31), dict(tq=1 << 30), dict(max_q=-1), dict(max_k=-1), dict(q=None),
              dict(k=None), dict(v=None), dict(q=P + 8), dict(k=P + 8), dict(v=P + 2), dict(q_row=63), dict(q_row=516),
              dict(k_row=1 << 23), dict(v_row=260), dict(k_head=4), dict(q_head=-64), dict(start_q=None),
              dict(start_k=None), dict(start_q=P + 2), dict(used_k=P + 1), dict(BIAS, rel_bucket=None),
              dict(BIAS, rel_buckets=0), dict(BIAS, rel_buckets=1025), dict(BIAS, rel_reach=-1),
              dict(BIAS, rel_reach=2000), dict(BIAS, rel_weight=P + 1)]
    for bad in shared:
        assert _attention_fwd(lib, **bad) == EINVAL, bad
        assert _attention_bwd(lib, **dict(bad, dw=P if "rel_weight" in bad else None)) == EINVAL, bad
    for bad in (dict(dtype=2), dict(head_dim=48), dict(head_dim=256), dict(BIAS, dtype=0), dict(BIAS, wdtype=5),
                dict(dtype=0, residue=P)):
        assert _attention_fwd(lib, **bad) == EDTYPE, bad
    for bad in (dict(out=None), dict(out=P + 8), dict(residue=P + 8), dict(lse=P + 2)):
        assert _attention_fwd(lib, **bad) == EINVAL, bad
    for bad in (dict(out=None), dict(lse=None), dict(do=None), dict(dq=None), dict(dk=None), dict(dv=None),
                dict(do=P + 8), dict(dk=P + 4), dict(dw=P), dict(BIAS), dict(residue=P + 8)):
        assert _attention_bwd(lib, **bad) == EINVAL, bad
    assert lib.lram_attention_forward(None, P, None, None, None, 0, None) == EINVAL
    n = ctypes.c_size_t(0)
    a = _describe()
    assert lib.lram_attention_backward_workspace_bytes(ctypes.byref(a), ctypes.byref(n)) == 0 and n.value >= 300 * 8 * 4
    for bad in (dict(ws=None), dict(ws=P + 4), dict(ws_bytes=n.value - 1)):
        assert _attention_bwd(lib, **bad) == EWORKSPACE, bad
    one = dict(tq=1, tk=100000, max_q=1, max_k=100000, batch=1)  # few rows: the keys are divided
    a = _describe(**one)
    assert lib.lram_attention_forward_workspace_bytes(ctypes.byref(a), ctypes.byref(n)) == 0 and n.value > 0
    for bad in (dict(ws=None), dict(ws=P + 4), dict(ws_bytes=n.value - 1)):
        assert _attention_fwd(lib, **one, **bad) == EWORKSPACE, bad
    assert lib.lram_attention_forward_workspace_bytes(ctypes.byref(a), None) == EINVAL
    assert _attention_fwd(lib, tq=0, q=None, out=None) == 0  # empty: nothing to do


def test_expected_lengths_past_the_tensors(lib):
    """The workspace of any expectation is that of the tensors' whole lengths at most."""
    n, want = ctypes.c_size_t(0), ctypes.c_size_t(0)
    for size in (lib.lram_attention_forward_workspace_bytes, lib.lram_attention_backward_workspace_bytes):
        assert size(ctypes.byref(_describe(max_q=300, max_k=300)), ctypes.byref(want)) == 0
        for longest in (301, 1 << 31, 1 << 40, (1 << 63) - 1):
            assert size(ctypes.byref(_describe(max_q=longest, max_k=longest)), ctypes.byref(n)) == 0
            assert n.value == want.value


@pytest.mark.parametrize("dtype,d,heads,reach", [(1, 128, 4, 1951), (0, 64, 4, 1951), (0, 128, 4, 586), (1, 64, 8, 927),
                                                 (1, 64, 256, 0)])
def test_the_longest_reach(lib, dtype, d, heads, reach):
    """What the header allows, and one more."""
    n = ctypes.c_size_t(0)
    for extra, rc in ((0, 0), (1, EINVAL)):
        a = _describe(**dict(BIAS, dtype=dtype, wdtype=dtype, head_dim=d, heads=heads, kv_heads=4, rel_reach=reach + extra,
                             q_row=heads * d, k_row=4 * d, v_row=4 * d))
        if heads == 256:  # 64 heads of a group leave no room for a table
            rc = EINVAL
        assert lib.lram_attention_forward_workspace_bytes(ctypes.byref(a), ctypes.byref(n)) == rc
        assert lib.lram_attention_backward_workspace_bytes(ctypes.byref(a), ctypes.byref(n)) == rc


@pytest.mark.parametrize("buckets,reach,both", [(32, 128, True), (32, 128, False), (8, 4, True), (16, 1000, False),
                                                (2, 1, True), (1, 1, False), (3, 40, False), (4, 3, True)])
def test_buckets_follow_their_definition(buckets, reach, both):
    got = lram.relative_buckets(buckets, reach, both, device="cpu").tolist()
    side = buckets // 2 if both else buckets
    near = max(side // 2, 1)
    for d, b in zip(range(-reach, reach + 1), got):
        a = abs(d) if both else max(-d, 0)
        base = side if both and d > 0 else 0
        if a < near:
            assert b == base + min(a, side - 1)
            continue
        want = near + (math.log(a / near) / math.log(reach / near) * (side - near) if reach > near else side)
        # at an exact power the quotient of rounded logarithms may fall on either side
        ok = {min(math.floor(want - 1e-9), side - 1), min(math.floor(want + 1e-9), side - 1)}
        assert b - base in ok, (d, b, want)
    assert got[reach] == 0 and min(got) >= 0 and max(got) < buckets
    assert got[0] == side - 1  # the longest distance takes the last bucket of its side


def test_buckets_and_plans_refuse():
    for bad in ((0, 4, True), (1, 4, True), (32, 7, True), (0, 4, False)):
        with pytest.raises(lram.LramError):
            lram.relative_buckets(*bad, device="cpu")
    for bad in (dict(queries=[1, 2], keys=[1]), dict(queries=[-1]), dict(queries=[1], keys=[9], capacity=8),
                dict(queries=[1 << 30, 1 << 30])):
        with pytest.raises(lram.LramError):
            lram.pack(device="cpu", **bad)


def test_plans():
    p = lram.pack([3, 0, 2], device="cpu")
    assert p.start_q.tolist() == p.start_k.tolist() == [0, 3, 3, 5] and (p.max_q, p.max_k) == (3, 3) and p.used_k is None
    p = lram.pack([1, 1], [7, 2], capacity=8, device="cpu")
    assert p.start_q.tolist() == [0, 1, 2] and p.start_k.tolist() == [0, 8, 16] and p.used_k.tolist() == [7, 2]
    assert (p.max_q, p.max_k) == (1, 7)
    p = lram.pack([], device="cpu")
    assert p.start_q.tolist() == [0] and p.max_q == 0


def test_binding_refuses_host_tensors():
    x, w = torch.zeros(2, 8), torch.ones(8)
    with pytest.raises(lram.LramError, match="GPU"):
        lram.layer_norm_forward(x, w, w)
    q = torch.zeros(2, 1, 32)
    with pytest.raises(lram.LramError, match="GPU"):
        lram.attention_forward(q, q, q, lram.pack([2], device="cpu"))


# The reference's own gradients, against differences of its forward.

def test_reference_norm_gradients_by_differences():
    g = torch.Generator().manual_seed(1)
    x, w, b = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((5, 7), (7,), (7,)))
    dy = torch.randn((5, 7), generator=g, dtype=torch.float64)
    ref.HALF[torch.float64] = 2.0 ** -53
    got = ref.norm(x, w, b, 1e-5, dy=dy)
    h = 1e-6
    for name, t in (("dx", x), ("dw", w), ("db", b)):
        for i in range(t.numel()):
            keep = t.view(-1)[i].item()
            side = []
            for s in (h, -h):
                t.view(-1)[i] = keep + s
                side.append((ref.norm(x, w, b, 1e-5)["y"][0] * dy).sum().item())
            t.view(-1)[i] = keep
            assert abs((side[0] - side[1]) / (2 * h) - got[name][0].view(-1)[i].item()) < 1e-6


@pytest.mark.parametrize("causal,nq,nk", [(True, [3, 4, 1], [3, 2, 5]), (False, [2, 0, 3], [4, 2, 0])])
def test_reference_attention_gradients_by_differences(causal, nq, nk):
    g = torch.Generator().manual_seed(2)
    ref.HALF[torch.float64] = 2.0 ** -53
    q = torch.randn((sum(nq), 4, 3), generator=g, dtype=torch.float64)
    k, v = (torch.randn((sum(nk), 2, 3), generator=g, dtype=torch.float64) for _ in range(2))
    w = torch.randn((4, 3), generator=g, dtype=torch.float64)
    do = torch.randn(q.shape, generator=g, dtype=torch.float64)
    bucket = torch.tensor([2, 0, 0, 1, 1])
    sq, sk = ([sum(n[:i]) for i in range(len(n))] for n in (nq, nk))

    def run(do=None):
        return ref.attention(q, k, v, nq, nk, sq, sk, causal, 0.7, w, bucket, do)

    got, h = run(do), 1e-6
    for name, t in (("dq", q), ("dk", k), ("dv", v), ("dw", w)):
        for i in range(t.numel()):
            keep = t.view(-1)[i].item()
            side = []
            for s in (h, -h):
                t.view(-1)[i] = keep + s
                side.append((run()["out"][0] * do).sum().item())
            t.view(-1)[i] = keep
            assert abs((side[0] - side[1]) / (2 * h) - got[name][0].view(-1)[i].item()) < 1e-6, (name, i)
