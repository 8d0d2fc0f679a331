"""What the autograd wrappers do with derivatives that they do not offer."""
import pytest
import torch
from torch.autograd import forward_ad

import paper_2107_03474_amd as lram

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _norm_inputs():
    return torch.randn((5, 64), device=DEV), torch.ones(64, device=DEV), torch.zeros(64, device=DEV)


def _attention_inputs():
    return [torch.randn((20, 2, 32), device=DEV) for _ in range(3)] + [lram.pack([20])]


def _lookup_inputs():
    return torch.rand((6, 8), device=DEV) * 4, torch.randn((4 ** 8, 32), device=DEV), (4,) * 8


def _theta_inputs():
    return torch.randn((6, 16), device=DEV), torch.randn((4 ** 8, 64), device=DEV), (4,) * 8


CALLS = [(lambda *a: lram.layer_norm(*a), _norm_inputs),
         (lambda x, *a: lram.layer_norm(x, *a, residual=torch.ones_like(x))[0], _norm_inputs),
         (lambda *a: lram.attention(*a), _attention_inputs),
         (lambda *a: lram.lookup(*a), _lookup_inputs), (lambda *a: lram.theta(*a), _theta_inputs)]
NAMES = ["norm", "norm-residual", "attention", "lookup", "theta"]


@pytest.mark.parametrize("call,inputs", CALLS, ids=NAMES)
def test_forward_mode_is_refused(call, inputs):
    x, *rest = inputs()
    with forward_ad.dual_level():
        with pytest.raises(NotImplementedError):
            call(forward_ad.make_dual(x, torch.ones_like(x)), *rest)
        call(x, *rest)  # no tangent: nothing to refuse


@pytest.mark.parametrize("call,inputs", CALLS, ids=NAMES)
def test_second_derivatives_are_refused(call, inputs):
    x, *rest = inputs()
    x.requires_grad_()
    first, = torch.autograd.grad(call(x, *rest).square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        first.sum().backward()
