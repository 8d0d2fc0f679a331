"""Tensors of the layer's operators that do not start on 16 bytes, as views into larger ones do."""
import pytest
import torch

import layer_reference as ref
import paper_2107_03474_amd as lram

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


def _randn(g, shape, dtype):
    return torch.randn(shape, generator=g, device=DEV).to(dtype)


def _off(t):
    """A copy of t one element behind a boundary of 16 bytes."""
    x = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)[1:].view(t.shape)
    x.copy_(t)
    assert x.is_contiguous() and x.data_ptr() % 16
    return x


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,width", [(6, 1021), (1, 7), (40, 64)])
def test_norm(rows, width, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    x, r, dy, dh = (_randn(g, (rows, width), dtype) for _ in range(4))
    w, b = _randn(g, (width,), dtype), _randn(g, (width,), dtype)
    want = ref.norm(x, w, b, 1e-5, r, dy, dh)
    y, h, mean, rstd = lram.layer_norm_forward(_off(x), w, b, residual=_off(r))
    dx, dw, db = lram.layer_norm_backward(_off(h), w, mean, rstd, _off(dy), grad_h=_off(dh))
    for n, t in dict(y=y, h=h, dx=dx, dw=dw, db=db).items():
        ref.assert_close(n, t, want[n])
    x2, w2 = _off(x).requires_grad_(), w.clone().requires_grad_()
    y = lram.layer_norm(x2, w2, b)
    y.backward(_off(dy))
    want = ref.norm(x, w, b, 1e-5, dy=dy)
    for n, t in dict(y=y.detach(), dx=x2.grad, dw=w2.grad).items():
        ref.assert_close(n, t, want[n])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_of_later_rows_and_a_gradient_through_cat(dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    x, dy = _randn(g, (8, 1021), dtype), _randn(g, (11, 1021), dtype)
    w, b = _randn(g, (1021,), dtype), _randn(g, (1021,), dtype)
    with torch.no_grad():
        assert torch.equal(lram.layer_norm(x[1:], w, b), lram.layer_norm(x, w, b)[1:])
    leaf = x.clone().requires_grad_()
    torch.cat([dy[:3] * 2, lram.layer_norm(leaf, w, b)]).backward(dy)
    ref.assert_close("dx", leaf.grad, ref.norm(x, w, b, 1e-5, dy=dy[3:])["dx"])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_gradient_of_attention_through_cat(dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    q, do = (_randn(g, (20, 2, 32), dtype) for _ in range(2))
    k, v = (_randn(g, (20, 1, 32), dtype) for _ in range(2))
    leaf = q.clone().requires_grad_()
    out = lram.attention(leaf, k, v, lram.pack([20]))
    torch.cat([torch.ones(1, dtype=dtype, device=DEV), out.flatten()]).backward(
        torch.cat([torch.ones(1, dtype=dtype, device=DEV), do.flatten()]))
    want = ref.attention(q, k, v, [20], [20], [0], [0], False, 32 ** -0.5, do=do)
    ref.assert_close("dq", leaf.grad, want["dq"])
