"""How attention divides its work where the expected lengths say little of the real ones: workspaces stay small, and no
launch grows with the pieces.  Host only."""
import ctypes

import pytest

from paper_2107_03474_amd import layer

P = 0x10000  # never dereferenced


def _bytes(**kw):
    a = layer._Attention(dtype=1, wdtype=1, heads=8, kv_heads=8, head_dim=64, batch=1, causal=0, scale=0.125, tq=1, tk=1,
                         max_q=1, max_k=1, q=P, k=P, v=P, q_row=512, q_head=64, k_row=512, k_head=64, v_row=512, v_head=64,
                         start_q=P, start_k=P)
    for n, v in kw.items():
        setattr(a, n, v)
    got, lib = [], layer._library()
    for size in (lib.lram_attention_forward_workspace_bytes, lib.lram_attention_backward_workspace_bytes):
        n = ctypes.c_size_t(0)
        assert size(ctypes.byref(a), ctypes.byref(n)) == 0
        got.append(n.value)
    return got


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("kv_heads", [1, 8])
@pytest.mark.parametrize("max_q,max_k", [(1, 1 << 20), (4, 1 << 20), (40, 1 << 20), (40, 5000), (0, 0), (1 << 20, 1)])
@pytest.mark.parametrize("rows", [1000, 100_000, 1_000_000])
def test_understated_lengths(rows, max_q, max_k, kv_heads, dtype):
    """The pieces of a call that is told of short sequences and gets long ones cost no more than those of one that is told:
    rows' own statistics, and partial results for about two rounds of workgroups, of 128 rows each."""
    heads, d = 8, 64
    forward, backward = _bytes(tq=rows, tk=rows, max_q=max_q, max_k=max_k, kv_heads=kv_heads, dtype=dtype, k_row=kv_heads * 64,
                               v_row=kv_heads * 64)
    rounds = 2048 * 2  # workgroups, and as many again for tiles that are not full
    assert forward <= rounds * 128 * (d + 1) * 4
    assert backward <= 2 * (rows * heads + 4) * 4 + rounds * 128 * 2 * d * 4


def test_honest_lengths_are_divided_as_before():
    """Few queries over many keys, few keys under many rows: pieces."""
    def pieces(heads=8, d=64, **kw):
        return _bytes(**kw)[0] // (kw["tq"] * heads * (d + 1) * 4)

    assert pieces(tq=1, tk=100_000, max_k=100_000) == 61              # 64 of 128 whole keys each, where 61 are enough
    assert pieces(tq=70, tk=20_000, max_q=70, max_k=20_000) == 20     # none shorter than 1,024 keys
    assert pieces(tq=32, tk=32 * 8192, batch=32, max_k=8192) == 2     # a round of 512 workgroups
    assert pieces(tq=5000, tk=5000, batch=3, max_q=3000, max_k=3000) == 2
    assert _bytes(tq=2000, tk=130, max_q=2000, max_k=130)[1] == (2 * 2000 * 8 + 2 * 130 * 8 * 2 * 64) * 4
