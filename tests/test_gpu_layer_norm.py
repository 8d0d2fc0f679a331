"""Layer norm on the GPU against the plain 64-bit form and its derived bounds (layer_reference.py)."""
import pytest
import torch

import layer_reference as ref
import paper_2107_03474_amd as lram

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


def _inputs(rows, width, dtype, wtype, seed=0, mean=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def randn(*s, scale=1.0):
        return torch.randn(s, generator=g, device=DEV) * scale

    x = (randn(rows, width, scale=2.0) + mean * randn(rows, 1)).to(dtype)
    r, dy, dh = (randn(rows, width).to(dtype) for _ in range(3))
    return x, r, dy, dh, (1 + randn(width, scale=0.3)).to(wtype), randn(width, scale=0.3).to(wtype)


def _check(x, r, dy, dh, w, b, eps=1e-5):
    y, h, mean, rstd = lram.layer_norm_forward(x, w, b, eps, residual=r)
    dx, dw, db = lram.layer_norm_backward(h, w, mean, rstd, dy, grad_h=dh)
    torch.cuda.synchronize()
    want = ref.norm(x, w, b, eps, r, dy, dh)
    got = dict(y=y, dx=dx, dw=dw, db=db)
    if r is not None:
        got["h"] = h
    else:
        assert h is x
    for n, t in got.items():
        assert t.dtype == (w.dtype if n in ("dw", "db") else x.dtype)
        ref.assert_close(n, t, want[n])


@pytest.mark.parametrize("dtype,wtype", [(F32, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("rows,width", [(1, 1), (3, 2), (1, 512), (5, 7), (4, 63), (9, 64), (2, 255), (6, 257), (33, 512),
                                        (7, 1021), (3, 2048), (5, 2049), (4, 4100), (2, 8192), (3, 8200), (2, 16384),
                                        (4097, 40), (9000, 129)])
def test_norm(rows, width, dtype, wtype):
    x, r, dy, dh, w, b = _inputs(rows, width, dtype, wtype, rows + width)
    _check(x, r, dy, dh, w, b)
    _check(x, None, dy, None, w, b)


def test_many_rows_share_a_workgroup():
    _check(*_inputs(70001, 96, BF16, BF16))
    _check(*_inputs(5001, 8192, BF16, F32))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [1024, 1025])
def test_waves_and_workgroups_share_a_width(rows, dtype):
    for width in (260, 900, 1021, 2001):
        _check(*_inputs(rows, width, dtype, dtype, width))


def test_without_gradients():
    x, r, dy, dh, w, b = _inputs(30, 96, BF16, F32)
    w.requires_grad_()
    with torch.no_grad():
        y, h = lram.layer_norm(x, w, b, residual=r)
        assert not y.requires_grad and torch.equal(lram.layer_norm(x, w, b), lram.layer_norm_forward(x, w, b)[0])
    y2, h2 = lram.layer_norm(x, w, b, residual=r)
    assert y2.requires_grad and torch.equal(y, y2) and torch.equal(h, h2)


def test_constant_rows_and_large_means():
    x, r, dy, dh, w, b = _inputs(40, 320, F32, F32, 3, mean=1000.0)  # variance far below the squared mean
    _check(x, None, dy, None, w, b)
    x = torch.full((3, 100), 7.0, device=DEV)
    y, h, mean, rstd = lram.layer_norm_forward(x, w[:100].contiguous(), b[:100].contiguous(), 1e-5)
    assert torch.equal(y, b[:100].expand(3, 100)) and torch.equal(mean, torch.full((3,), 7.0, device=DEV))


def test_a_row_with_nan_or_inf_stays_alone():
    x, r, dy, dh, w, b = _inputs(6, 200, BF16, BF16)
    x[2, 5] = float("nan")
    x[4, 0] = float("inf")
    y, h, mean, rstd = lram.layer_norm_forward(x, w, b, residual=r)
    assert torch.isnan(y[2]).all() and torch.isnan(y[4]).all()
    keep = [0, 1, 3, 5]
    ref.assert_close("y", y[keep], ref.norm(x[keep], w, b, 1e-5, r[keep])["y"])


def test_rows_past_32_bits():
    rows, width = 65537, 32 * 1024 // 2
    x = torch.zeros((rows, width), dtype=F32, device=DEV)       # 4.3 GB: the last rows lie past 2^32 bytes
    w, b = torch.ones(width, device=DEV), torch.zeros(width, device=DEV)
    x[-3:] = torch.randn((3, width), device=DEV)
    y, h, mean, rstd = lram.layer_norm_forward(x, w, b)
    ref.assert_close("y", y[-3:], ref.norm(x[-3:], w, b, 1e-5)["y"])
    dx, dw, db = lram.layer_norm_backward(h, w, mean, rstd, x)
    ref.assert_close("dx", dx[-3:], ref.norm(x[-3:], w, b, 1e-5, dy=x[-3:])["dx"])


def test_leading_dimensions_and_empty():
    x, r, dy, dh, w, b = _inputs(24, 72, BF16, BF16)
    shape = (2, 3, 4, 72)
    y, h, mean, rstd = lram.layer_norm_forward(x.view(shape), w, b, residual=r.view(shape))
    y2, h2, _, _ = lram.layer_norm_forward(x, w, b, residual=r)
    assert y.shape == shape and mean.shape == shape[:-1] and torch.equal(y.view(24, 72), y2) and torch.equal(h.view(24, 72), h2)
    e = x[:0]
    y, h, mean, rstd = lram.layer_norm_forward(e, w, b)
    dx, dw, db = lram.layer_norm_backward(h, w, mean, rstd, e)
    assert y.shape == (0, 72) and dx.shape == (0, 72) and not dw.any() and not db.any()


def test_gradients_without_the_weights():
    x, r, dy, dh, w, b = _inputs(50, 130, F32, F32)
    y, h, mean, rstd = lram.layer_norm_forward(x, w, b)
    dx, dw, db = lram.layer_norm_backward(h, w, mean, rstd, dy, want_grad_weight=False)
    assert dw is None and db is None
    assert torch.equal(dx, lram.layer_norm_backward(h, w, mean, rstd, dy)[0])


@pytest.mark.parametrize("residual", [False, True])
def test_autograd(residual):
    x, r, dy, dh, w, b = _inputs(30, 96, F32, F32)
    leaves = [t.clone().requires_grad_() for t in (x, r, w, b)]
    if residual:
        y, h = lram.layer_norm(leaves[0], leaves[2], leaves[3], residual=leaves[1])
        (y * dy).sum().backward(retain_graph=True)
        first = leaves[0].grad.clone()
        for t in leaves:
            t.grad = None
        ((y * dy).sum() + (h * dh).sum()).backward()
        ref.assert_close("dx", leaves[0].grad, ref.norm(x, w, b, 1e-5, r, dy, dh)["dx"])
        ref.assert_close("dx", first, ref.norm(x, w, b, 1e-5, r, dy)["dx"])
        assert torch.equal(leaves[1].grad, leaves[0].grad)
        for t in leaves:
            t.grad = None
        y, h = lram.layer_norm(leaves[0], leaves[2], leaves[3], residual=leaves[1])
        (h * dh).sum().backward()   # nothing reaches the norm itself
        assert torch.equal(leaves[0].grad, dh) and leaves[2].grad is None
    else:
        y = lram.layer_norm(leaves[0], leaves[2], leaves[3])
        (y * dy).sum().backward()
        want = ref.norm(x, w, b, 1e-5, dy=dy)
        for n, t in (("dx", leaves[0]), ("dw", leaves[2]), ("db", leaves[3])):
            ref.assert_close(n, t.grad, want[n])


def test_gradients_by_differences():
    """Directional differences of the kernel's own forward, in fp32, against its gradients: the forward's bounded errors
    over the step, and the third-order term taken from the 64-bit form's differences at the same step."""
    x, r, dy, dh, w, b = _inputs(8, 100, F32, F32)
    y, h, mean, rstd = lram.layer_norm_forward(x, w, b)
    grads = lram.layer_norm_backward(h, w, mean, rstd, dy)
    step = 2.0 ** -6
    for k, (t, g) in enumerate(zip((x, w, b), grads)):
        d = torch.sign(torch.randn_like(t))
        side, side64, slack = [], [], 0.0
        for s in (step, -step):
            args = [x, w, b]
            args[k] = (t + s * d)
            yk = lram.layer_norm_forward(*args)[0]
            y64, bound = ref.norm(*args, 1e-5)["y"]
            side.append(float((yk.double() * dy.double()).sum()))
            side64.append(float((y64 * dy.double()).sum()))
            slack += float((bound * dy.double().abs()).sum())
        want = ref.norm(x, w, b, 1e-5, dy=dy)[("dx", "dw", "db")[k]]
        along, along64 = float((g.double() * d.double()).sum()), float((want[0] * d.double()).sum())
        curved = (side64[0] - side64[1]) / (2 * step) - along64
        # (t + s d) is itself rounded: half a unit of |t|, along the gradient
        moved = float(((2.0 ** -24) * (t.abs() + step).double() * want[0].abs()).sum()) * 2 / (2 * step)
        assert abs((side[0] - side[1]) / (2 * step) - curved - along) <= slack / (2 * step) + moved + float(want[1].sum())


def test_same_bits_every_time_and_in_a_graph():
    x, r, dy, dh, w, b = _inputs(3000, 520, BF16, BF16)

    def step():
        y, h, mean, rstd = lram.layer_norm_forward(x, w, b, residual=r)
        return (y, h, *lram.layer_norm_backward(h, w, mean, rstd, dy, grad_h=dh))

    first = step()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for seed in range(3):
        n = _inputs(3000, 520, BF16, BF16, seed + 5)
        for t, v in zip((x, r, dy, dh, w, b), n):
            t.copy_(v)
        eager = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(eager, captured))
        assert all(torch.equal(a, c) for a, c in zip(eager, step()))
    assert len(first) == 5


def test_refuses():
    x, r, dy, dh, w, b = _inputs(4, 64, BF16, BF16)
    for bad in (dict(x=x.t()), dict(x=x.half()), dict(weight=w[:32]), dict(weight=w.half(), bias=b.half()),
                dict(bias=b.float()), dict(residual=r[:2]), dict(residual=r.float()), dict(x=x.cpu()),
                dict(weight=w.cpu(), bias=b.cpu()), dict(x=x[:, :0]), dict(eps=-1.0),
                dict(x=torch.zeros(2, 16385, device=DEV), weight=torch.zeros(16385, device=DEV),
                     bias=torch.zeros(16385, device=DEV), residual=None)):
        with pytest.raises(lram.LramError):
            lram.layer_norm_forward(**dict(dict(x=x, weight=w, bias=b, residual=None), **bad))
    y, h, mean, rstd = lram.layer_norm_forward(x, w, b)
    for bad in (dict(mean=mean[:2]), dict(rstd=rstd.double()), dict(grad_y=dy.float()), dict(grad_h=dh[:1])):
        with pytest.raises(lram.LramError):
            lram.layer_norm_backward(**dict(dict(h=h, weight=w, mean=mean, rstd=rstd, grad_y=dy), **bad))
    with pytest.raises(lram.LramError, match="workspace"):
        big = torch.zeros((9000, 64), dtype=BF16, device=DEV)
        y, h, mean, rstd = lram.layer_norm_forward(big, w, b)
        lram.layer_norm_backward(h, w, mean, rstd, big, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
