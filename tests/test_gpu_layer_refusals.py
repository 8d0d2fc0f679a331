"""What the layer's refusals say."""
import pytest
import torch

import paper_2107_03474_amd as lram

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("d", [16, 48, 80, 96, 256])
def test_head_width(d):
    q = torch.zeros((4, 2, d), device=DEV)
    for call in (lambda: lram.attention_forward(q, q, q, lram.pack([4])), lambda: lram.attention(q, q, q, lram.pack([4]))):
        with pytest.raises(lram.LramError, match="head_dim must be 32, 64 or 128"):
            call()


def test_bias_of_too_many_distances():
    for heads, reach in ((16, 128), (1, 1952), (64, 0)):
        q, k = torch.zeros((4, heads, 64), device=DEV), torch.zeros((4, 1, 64), device=DEV)
        rel = lram.RelativeBias(torch.zeros((heads, 32), device=DEV), torch.zeros(2 * reach + 1, dtype=torch.int32, device=DEV))
        with pytest.raises(lram.LramError, match="2 reach"):
            lram.attention_forward(q, k, k, lram.pack([4]), rel=rel)
    q = torch.zeros((4, 1, 128), device=DEV)
    rel = lram.RelativeBias(torch.zeros((1, 32), device=DEV), torch.zeros(2 * 587 + 1, dtype=torch.int32, device=DEV))
    with pytest.raises(lram.LramError, match="2 reach"):
        lram.attention_forward(q, q, q, lram.pack([4]), rel=rel)
    rel = lram.RelativeBias(torch.zeros((1, 257), device=DEV), torch.zeros(9, dtype=torch.int32, device=DEV))
    with pytest.raises(lram.LramError, match="256 buckets"):
        lram.attention_forward(q, q, q, lram.pack([4]), rel=rel)


def test_what_does_not_lie_on_16_bytes():
    x = torch.zeros((8, 2, 72), dtype=torch.bfloat16, device=DEV)
    k = torch.zeros((8, 2, 64), dtype=torch.bfloat16, device=DEV)
    wide = torch.zeros((8, 2, 68), dtype=torch.bfloat16, device=DEV)
    for q in (x[..., 4:68], wide[..., :64], k[:1].expand(8, 2, 64)):
        with pytest.raises(lram.LramError, match="16 bytes"):
            lram.attention_forward(q, k, k, lram.pack([8]))


def test_heads_and_scale():
    q, k = torch.zeros((4, 6, 32), device=DEV), torch.zeros((4, 4, 32), device=DEV)
    with pytest.raises(lram.LramError, match="multiple of k's"):
        lram.attention_forward(q, k, k, lram.pack([4]))
    q, k = torch.zeros((4, 65, 32), device=DEV), torch.zeros((4, 1, 32), device=DEV)
    with pytest.raises(lram.LramError, match="64 times"):
        lram.attention_forward(q, k, k, lram.pack([4]))
    with pytest.raises(lram.LramError, match="scale"):
        lram.attention_forward(k, k, k, lram.pack([4]), scale=-1.0)


def test_norm_of_wide_rows_and_negative_eps():
    for width, eps, what in ((16385, 1e-5, "16384"), (64, -1.0, "eps")):
        x, w = torch.zeros((2, width), device=DEV), torch.zeros(width, device=DEV)
        with pytest.raises(lram.LramError, match=what):
            lram.layer_norm_forward(x, w, w, eps)
