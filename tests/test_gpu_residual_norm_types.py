"""The type of h where no branch gives it: in the backward pass without h's gradient it is still the forward call's."""
import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300.layers import ResidualNorm

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("pre", ["rms", "layer"])
def test_only_u_is_used(pre, dtype):
    op = ResidualNorm(96, pre=pre, residual_scale=0.5)
    x = torch.randn(7, 96, device="cuda").requires_grad_()
    w = torch.ones(96, dtype=dtype, device="cuda").requires_grad_()
    u, h = op(x, pre_weight=w, dtype=dtype)
    assert u.dtype is torch.float32 and h.dtype is dtype
    du = torch.randn(7, 96, device="cuda")
    dx, dw = torch.autograd.grad(u, (x, w), du)
    assert torch.equal(dx, 0.5 * du) and dw.dtype is dtype and torch.equal(dw, torch.zeros_like(w))
    _, _, stats = op.forward(x.detach(), pre_weight=w.detach(), dtype=dtype)
    for stream in (None, torch.cuda.current_stream()):
        g = op.backward(du, None, x.detach(), pre_weight=w.detach(), stats=stats, dtype=dtype, stream=stream)
        assert torch.equal(g.x, dx) and torch.equal(g.pre_weight, dw)


def test_another_type_of_the_gradient_is_refused():
    op = ResidualNorm(96)
    x = torch.randn(7, 96, device="cuda")
    _, _, stats = op.forward(x, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        op.backward(None, torch.zeros(7, 96, dtype=torch.float16, device="cuda"), x, stats=stats, dtype=torch.bfloat16)
