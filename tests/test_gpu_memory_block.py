"""The transformer layer around the memory: its parts against plain 64-bit forms, training, and serving piece by piece."""
import pytest
import torch

import layer_reference as ref
import paper_2107_03474_amd as lram
from paper_2107_03474_amd.memory_block import KeyValueCache, MemoryBlock

pytestmark = pytest.mark.gpu
DEV = "cuda"
K = (4,) * 8


def _block(causal, w=128, heads=4, kv_heads=2, dtype=torch.float32):
    torch.manual_seed(3)
    b = MemoryBlock(w, heads, K, kv_heads, causal, buckets=16, reach=20, table_dtype=dtype, dtype=dtype)
    with torch.no_grad():
        b.bias.normal_()
        for p in list(b.norm_w) + list(b.norm_b):
            p.add_(0.2 * torch.randn_like(p))
        b.memory.table.normal_()
    return b


@pytest.mark.parametrize("causal", [False, True])
def test_layer_is_its_formula(causal):
    b = _block(causal).eval()
    lengths = [17, 1, 60]
    x = torch.randn((78, 128), device=DEV)
    got = b(x, lram.pack(lengths))
    with torch.no_grad():
        # the projections in 64 bits, the attention and the norms in their 64-bit forms; the memory is the module's own
        p = torch.nn.functional.linear(x.double(), b.qkv.weight.double(), b.qkv.bias.double()).float()
        q, k, v = p[:, :128].unflatten(1, (4, 32)), p[:, 128:192].unflatten(1, (2, 32)), p[:, 192:].unflatten(1, (2, 32))
        a = ref.attention(q, k, v, lengths, lengths, [0, 17, 18], [0, 17, 18], causal, 32 ** -0.5, b.bias, b.bucket)["out"][0]
        a = torch.nn.functional.linear(a.flatten(1), b.proj.weight.double(), b.proj.bias.double()).float()
        y = ref.norm(a, b.norm_w[0], b.norm_b[0], 1e-5, x)["y"][0].float()
        y = ref.norm(b.memory(y), b.norm_w[1], b.norm_b[1], 1e-5, y)["y"][0]
    # fp32 projections of 128 terms on values of a few units, through three normalised layers
    assert (got.double() - y).abs().max() < 2e-4


def test_training_step_reaches_every_parameter():
    b = _block(False, dtype=torch.float32).train()
    x = torch.randn((96, 128), device=DEV)
    target = torch.randn((96, 128), device=DEV)
    seqs = lram.pack([40, 56])
    opt = torch.optim.SGD([p for p in b.parameters()], lr=0.05)
    losses = []
    for _ in range(5):
        opt.zero_grad()
        loss = ((b(x, seqs) - target) ** 2).mean()
        loss.backward()
        if not losses:
            for n, p in b.named_parameters():
                assert p.grad is not None and bool(torch.isfinite(p.grad).all()) and bool(p.grad.any()), n
        opt.step()
        losses.append(float(loss))
    assert losses[-1] < losses[0]


def test_serving_piece_by_piece_is_the_whole():
    b = _block(True).eval()
    lengths = [21, 9]
    x = torch.randn((30, 128), device=DEV)
    with torch.no_grad():
        whole = b(x, lram.pack(lengths))
    cache = KeyValueCache(2, 32, 2, 32, torch.float32)
    rows = {0: x[:21], 1: x[21:]}
    want = {0: whole[:21], 1: whole[21:]}
    done = [0, 0]
    for step in ([12, 3], [1, 1], [5, 0], [3, 5]):
        piece = torch.cat([rows[s][done[s]:done[s] + n] for s, n in enumerate(step)])
        got = b.serve(piece, lram.pack(step), cache)
        expect = torch.cat([want[s][done[s]:done[s] + n] for s, n in enumerate(step)])
        # the same formula from other tiles: fp32 sums in another order
        assert (got - expect).abs().max() < 2e-4
        done = [d + n for d, n in zip(done, step)]
    assert done == lengths and cache.used.tolist() == lengths
    with pytest.raises(ValueError):
        _block(False).serve(x, lram.pack(lengths), cache)


def test_bf16_layer():
    b = _block(True, dtype=torch.bfloat16).train()
    x = torch.randn((70, 128), device=DEV).to(torch.bfloat16).requires_grad_()
    y = b(x, lram.pack([70]))
    y.float().square().mean().backward()
    assert y.dtype == torch.bfloat16 and bool(torch.isfinite(y.float()).all()) and bool(x.grad.any())
